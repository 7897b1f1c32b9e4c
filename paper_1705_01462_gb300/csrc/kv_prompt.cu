// Attention over the 4-bit cache, many query rows (prompts, chunks of prompts, drafts to verify): bf16 and
// fp16, on tcgen05.
//
// A block takes NQT tiles of 128 query rows (query, head of the group) of one (sequence, kv head) and a
// chunk of its tokens, BN at a time:
//   S[128 x BN] = Q K^T        K K-major in shared memory (128-byte swizzle), Q the TMEM operand; fp32 S in TMEM
//   P = 2^(x - r)              one thread a row, 64 tokens (a unit) at a time; P as fp16 over S in TMEM
//   O[128 x D] += P V          P the TMEM operand, V as it lies, token by token: the MN-major operand
// K and V are dequantized once per block into shared memory as fp16, so that a value costs its share of
// 128 NQT rows' arithmetic.  Queries in TMEM are not read from shared memory again with every tile of keys (32 rows of 32
// sequences of 2000 tokens, heads of 64 values: 53.5 us, and 57.5 from shared memory; of 128: 69.7 and 75.7); two
// tiles of rows of 128 values leave no columns for them.  BN = 128 where it fits: an MMA of N = 64 takes nearly as
// long as one of 128 (with BN = 64, 67.8 and 80.6 us there).  While a tile of rows does its softmax the other
// one's products run (NQT = 2), or the next scores into a second buffer (NQT = 1).
//
// Range.  Queries are scaled by a power of two per row; K and V by a power of two per 16 tokens (2^-ek,
// 2^-ev) that brings their largest magnitude below 2^15, at most a factor of 64, and each dequantizing warp works by
// itself.  S is multiplied by 2^ek; P takes 2^ev: p = 2^(x + ev - r) against V 2^-ev, and l sums p 2^-ev.  r is
// a row's largest x + ev at its last move, less 6, kept as its x and its ev (er), as a large x has no room for ev.  It moves
// only when exceeded by 14 - 6 = 8 (as in kv_attention.cuh), and only then is O rescaled, after the products that add to
// it.  Past scores of 4096 the differences x - r come before anything is added (`big`): in one multiply-add with the
// rounded reference, scores past 2^25 would turn into infinities or zeros.  `big` also stands for references of values past
// 2^33, beside which the exponents of zeros and far smaller values are raised, so that their p stays above 2^-126.
// What is rounded: lo + s c and probabilities to fp16 (11 bits); sums and statistics are fp32.  For bf16 outputs that is
// an eighth of the output's own rounding (1.67e-3 of the output in all, 1.66e-3 the output's alone).  For fp16 outputs the
// probabilities' would weigh as much as the output's (3.3e-4 in all, where the output's alone is 2.1e-4), so they take a second
// fp16 part in the other half of their scores' columns, and a second product with V (TWO): 262 us instead of 216 with the
// queries below, 42 instead of 39 with 36 rows of 256 values.  Keys and values remain: 2.1e-4 in all where keys are of one
// size, 2.2e-4 to 2.9e-4 where some of their dimensions are six times as large as the others.
//
// What bounds it, 2 x 1024 queries of 32 heads over 4096 to 6144 tokens, 8 kv heads of 128 values, 216 us where the products
// alone are due 92: tensor pipe 34% busy, ALU 46%, shared memory 39% of the time.  A tile of rows waits for
// its next scores for a third of the time, as TMEM has room for one buffer of them beside the sums; a block's
// start (8 us) and the second, partial wave of blocks are the rest.  36 rows of 256 values in a window of 4096: 39 us,
// dequantization (12 values a clock and SM) and the block's start.
//
// Warp roles (one block per SM): warps 0 .. 4 NQT - 1 softmax (TMEM lane = row); the next eight dequantize,
// in two groups that take units in turn, 16 tokens a warp; the last group of four holds the MMA issuer, which
// also allocates TMEM (converged, an elected lane issues: from a divergent lane an MMA took 100 clocks, 244 us).
// Every wait is bounded; on expiry FGQ_ERR_TIMEOUT is recorded, the roles leave their loops, MMAs in
// flight are waited for, and TMEM is freed.
#include "kv_attention.cuh"
#include "tc_common.cuh"

namespace fgq {
namespace {

using namespace dec;
using tc::sw128;

constexpr int PR_UN = 64;          // tokens of a unit: a softmax step, a dequantizing group's step
constexpr int PR_DEQ = 4;          // dequantizing warps of a group
constexpr int PR_GROUPS = 2;       // groups of them, taking units in turn
constexpr int PR_E = 16;           // units whose scales are kept: more than any role is ahead of another

template <int D, int NQT>
struct PrCfg {
  static constexpr int BN = D == 256 ? 64 : 128, H = BN / PR_UN;  // tokens and units of a tile
  static constexpr int NSB = NQT == 2 ? 1 : 2;                    // S buffers of a tile of rows
  // TMEM: NQT x NSB score buffers, NQT x D sums, and NQT x D / 2 words of queries where there is room
  static constexpr uint32_t O_COL = NQT * NSB * BN, Q_COL = O_COL + NQT * D;
  static constexpr bool QT = Q_COL + NQT * D / 2 <= 512;
  static constexpr uint32_t COLS = Q_COL + (QT ? NQT * D / 2 : 0) <= 256 ? 256 : 512;
  static constexpr int STAGES = D == 128 && !QT ? 2 : 3;
  static constexpr int Q_TILE = 128 * D * 2, KV_TILE = BN * D * 2;
  static constexpr int SMEM_Q = QT ? 0 : NQT * Q_TILE;
  static constexpr int SMEM = 1024 + SMEM_Q + 2 * STAGES * KV_TILE;
  static constexpr int DEQ0 = 4 * NQT, MMA = DEQ0 + PR_GROUPS * PR_DEQ;
  static constexpr int THREADS = 32 * (MMA + 4);
};

// Registers a thread of the softmax, dequantizing and MMA warpgroups: the last gives up what the others take
// over the launch's 96 (NQT = 2, 640 threads) or 128 (512).
template <int NQT>
struct PrRegs {
  static constexpr int LAUNCH = NQT == 2 ? 96 : 128, SOFTMAX = NQT == 2 ? 104 : 128, DEQ = NQT == 2 ? 104 : 160, MMA = 64;
  static_assert(128 * NQT * SOFTMAX + 256 * DEQ + 128 * MMA <= (128 * NQT + 384) * LAUNCH, "the launch's registers");
  static_assert(SOFTMAX >= LAUNCH && DEQ >= LAUNCH && MMA <= LAUNCH, "inc, inc, dec");
};

// Byte offset of 16-byte piece c (eight values) of row r in a tile of `rows` rows of D fp16: sub-tiles of 64
// columns, 128-byte swizzle.
__device__ __forceinline__ uint32_t tile_off(int r, int c, int rows) { return (uint32_t)((c >> 3) * rows * 128) + sw128(r, c & 7); }

// The MN-major operand with the 128-byte swizzle: 64 columns (128 bytes) of 8 k-rows make an atom of 1024
// bytes, the next 8 k-rows follow, lbo bytes lead to the next 64 columns.
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// D[tmem] (+)= A[tmem] * B[smem], fp16 operands.
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16_u(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

// The codes in the low nibbles of w's halves as fp16, by way of 1024 + c, and the next ones, of 64 + c.
__device__ __forceinline__ uint32_t codes2(uint32_t w) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"((w & 0x000f000fu) | 0x64006400u), "r"(0x64006400u));
  return r;
}
__device__ __forceinline__ uint32_t codes2_hi(uint32_t w) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"((w & 0x00f000f0u) | 0x54005400u), "r"(0x54005400u));
  return r;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

// N consecutive words of global memory, aligned as they come together (8 or 16 bytes at most).
template <int N>
__device__ __forceinline__ void ldg_words(const void* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = __ldg(static_cast<const uint32_t*>(p));
  } else if constexpr (N == 2) {
    const uint2 v = __ldg(static_cast<const uint2*>(p));
    w[0] = v.x, w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = __ldg(static_cast<const uint4*>(p) + i / 4);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  }
}

// A thread's NB pieces of eight values (piece 4 j + u of row `row`) from codes `w` to fp16 in a tile of BN rows.
template <int NB, int NG, int BN>
__device__ __forceinline__ void convert_row(uint32_t tile, int row, int u, const uint32_t (&w)[NB], const uint32_t (&par)[NG],
                                            float f) {
  uint32_t s2[NG], l2[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const float l = __uint_as_float(par[i] & 0xffff0000u) * f, s = __uint_as_float(par[i] << 16) * f;
    s2[i] = h2(s, s);
    l2[i] = h2(l, l);
  }
  const uint32_t at = tile + (uint32_t)((row >> 3) * 1024 + (row & 7) * 128);
  const uint32_t sw[2] = {at + (uint32_t)((u ^ (row & 7)) << 4), at + (uint32_t)(((4 + u) ^ (row & 7)) << 4)};
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int gi = j * NG / NB;
    const uint32_t x = w[j], y = w[j] >> 8;
    const uint32_t a = hfma2(codes2(x), s2[gi], l2[gi]), b = hfma2(codes2_hi(x), s2[gi], l2[gi]);
    const uint32_t c = hfma2(codes2(y), s2[gi], l2[gi]), d = hfma2(codes2_hi(y), s2[gi], l2[gi]);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sw[j & 1] + (uint32_t)((j >> 1) * BN * 128)), "r"(a),
                 "r"(b), "r"(c), "r"(d)
                 : "memory");
  }
}

// TWO: probabilities as two fp16 parts.
template <int D, int G, int NQT, bool TWO>
__global__ void __launch_bounds__(PrCfg<D, NQT>::THREADS, 1) kv_prompt_kernel(const __grid_constant__ AttnArgs a) {
  using C = PrCfg<D, NQT>;
  constexpr int S = C::STAGES, NB = D / 32, NG = D / G, ROWS = 128 * NQT, BN = C::BN, H = C::H, NSB = C::NSB;
  extern __shared__ uint8_t smem_pr[];
  __shared__ uint64_t k_full[S], k_empty[S], v_full[S], v_empty[S], s_full[NQT][NSB], q_full, drain_bar;
  __shared__ uint64_t p_full[NQT][2], pv_done[NQT][2];  // by the unit's parity
  __shared__ uint32_t tmem_slot, abort_word;
  __shared__ __align__(16) float e_k[PR_E][PR_DEQ];  // 2^ek of each 16 tokens
  __shared__ __align__(16) float e_v[PR_E][PR_DEQ], e_u[PR_E][PR_DEQ];  // ev, 2^-ev
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_pr) + 1023) & ~uintptr_t(1023));
  uint8_t* kbuf = smem + C::SMEM_Q;
  uint8_t* vbuf = kbuf + S * C::KV_TILE;
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t tmo = a.timeout_ns;

  int id = blockIdx.x;
  const int ch = id % a.chunks;
  id /= a.chunks;
  const int rt = id % a.row_tiles;
  id /= a.row_tiles;
  const int head = id % a.c.kv_heads;
  const int b = id / a.c.kv_heads;
  const int r0 = rt * ROWS;
  const int n = seq_len(a, b);
  const int nq = a.q_lens ? min(__ldg(a.q_lens + b), a.T) : a.T;
  int first, end;
  visible(a, n, nq, r0 / a.group, (min(r0 + ROWS, a.rows) - 1) / a.group, first, end);
  const int seen = first;  // tokens before it share its block of 16 and may never have been written
  first &= ~15;
  const int64_t lo64 = (int64_t)first + (int64_t)ch * a.chunk;
  const int lo = lo64 < end ? (int)lo64 : end;
  const int hi = ch == a.chunks - 1 ? end : (int)min((int64_t)end, lo64 + a.chunk);
  if (lo >= hi) {
    if (a.chunks == 1) {
      for (int i = threadIdx.x; i < ROWS * D; i += C::THREADS) {
        const int r = r0 + i / D;
        if (r >= a.rows) break;
        const int qi = r / a.group, h = r - qi * a.group;
        store_out(a, (((int64_t)b * a.T + qi) * a.q_heads + (int64_t)head * a.group + h) * D + i % D, 0.0f);
      }
    }
    return;
  }
  const int tiles = (hi - lo + BN - 1) / BN, units = tiles * H;

  pdl_trigger();  // the join may be brought up; it waits for this kernel's end
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&k_full[i], PR_DEQ * H);
      mbar_init(&v_full[i], PR_DEQ * H);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int q = 0; q < NQT; ++q) {
      for (int i = 0; i < NSB; ++i) mbar_init(&s_full[q][i], 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&p_full[q][i], 4);
        mbar_init(&pv_done[q][i], 1);
      }
    }
    mbar_init(&q_full, 4 * NQT);
    mbar_init(&drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == C::MMA) {
    tmem_alloc(&tmem_slot, C::COLS);
    tmem_relinquish();
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  auto fail = [&]() {
    *abort_flag = 1;
    record_error(a.err, FGQ_ERR_TIMEOUT);
  };

  // ------------------------------------------------------------------ dequantization
  if (warp >= C::DEQ0 && warp < C::MMA) {
    setmaxnreg_inc<PrRegs<NQT>::DEQ>();
    const int grp = (warp - C::DEQ0) / PR_DEQ, dw = (warp - C::DEQ0) % PR_DEQ;
    const int tr = lane & 7, u = lane >> 3;  // token of eight, quarter of its row
    constexpr int WPT = NB;                  // 32-bit words of codes a thread takes of a row
    const int32_t* table = a.c.table + (int64_t)b * a.c.max_pages;
    // 16 tokens' codes and parameters, two tokens a thread (tr and tr + 8), loaded a step ahead
    uint32_t kw[2][WPT], vw[2][WPT], kp[2][NG], vp[2][NG], kn[2][NG], vn[2][NG];
    const uint8_t* const kc0 = a.c.k_codes + tr * (D / 2) + u * 4 * WPT;
    const uint8_t* const vc0 = a.c.v_codes + tr * (D / 2) + u * 4 * WPT;
    const uint32_t *const kp0 = a.c.k_params + tr * NG, *const vp0 = a.c.v_params + tr * NG;
    int page = -1, slot = 0;
    bool in = false;
    auto look_up = [&](int un) {  // the page of this warp's 16 tokens of unit un
      const int tok = lo + un * PR_UN + 16 * dw;
      in = un < units && tok < hi;
      if (!in) return;
      const uint32_t pi = page_of(a.c, (uint32_t)tok);
      slot = tok - (int)pi * a.c.page_size;
      page = __ldg(table + pi);
    };
    // the lines of 16 tokens' codes and parameters on their way to L2: with rows of 128 bytes the loads a step
    // ahead are still waited for (8 rows of 256 values, 32 sequences of 2000 tokens: 113 us, and 103 with this), with
    // shorter ones they are not (128 values: 60.5 us, and 63.8)
    auto prefetch = [&]() {
      if (D < 256 || !in || page < 0 || page >= a.c.pages) return;
      constexpr int LC = D / 16;  // lines of 16 rows of codes
      const int64_t r = ((int64_t)page * a.c.kv_heads + head) * a.c.page_size + slot;
      const uint8_t* c = (lane & LC ? a.c.v_codes : a.c.k_codes) + r * (D / 2) + (lane & (LC - 1)) * 128;
      const uint32_t* p = (lane & 1 ? a.c.v_params : a.c.k_params) + r * NG + (lane >> 1) * 32;
      if (lane < 2 * LC) asm volatile("prefetch.global.L2 [%0];" ::"l"(c));
      if (lane < (NG > 2 ? NG : 2)) asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
    };
    int64_t row0 = 0;
    bool good = false;
    auto locate = [&]() {
      good = in && page >= 0 && page < a.c.pages;
      if (in && !good && lane == 0) record_error(a.err, FGQ_ERR_ARG);
      row0 = ((int64_t)page * a.c.kv_heads + head) * a.c.page_size + slot;
    };
    // parameters, zeros for tokens that were never written (so their values are 0 whatever the codes)
    auto params = [&](const uint32_t* p0, int un, uint32_t (&p)[2][NG]) {
      const int tok = lo + un * PR_UN + 16 * dw + tr;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < NG; ++i) p[k][i] = 0u;
        if (good && tok + 8 * k < hi && tok + 8 * k >= seen) ldg_words<NG>(p0 + row0 * NG + 8 * k * NG, p[k]);
      }
    };
    auto codes = [&](const uint8_t* c0, uint32_t (&w)[2][WPT]) {  // of the block's rows, which lie in one page
      if (!good) return;
#pragma unroll
      for (int k = 0; k < 2; ++k) ldg_words<WPT>(c0 + row0 * (D / 2) + 8 * k * (D / 2), w[k]);
    };
#pragma unroll
    for (int i = 0; i < WPT; ++i) kw[0][i] = kw[1][i] = vw[0][i] = vw[1][i] = 0u;
    look_up(grp);
    locate();
    params(kp0, grp, kp);
    params(vp0, grp, vp);
    codes(kc0, kw);
    codes(vc0, vw);
    look_up(grp + PR_GROUPS);
    bool ok = tmo != 0;
#pragma unroll 1
    for (int un = grp; un < units; un += PR_GROUPS) {
      const int it = un / H, st = it % S;
      // the largest |lo| and s of the 16 tokens' keys and values, as bf16 bits: every |value| is below
      // 2 max(|lo|, 16 s) < 2^(ek + 15)
      uint32_t mk = 0u, mv = 0u;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          mk = __vmaxu2(mk, kp[k][i] & 0x7fff7fffu);
          mv = __vmaxu2(mv, vp[k][i] & 0x7fff7fffu);
        }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        mk = __vmaxu2(mk, __shfl_xor_sync(FULL_MASK, mk, o));
        mv = __vmaxu2(mv, __shfl_xor_sync(FULL_MASK, mv, o));
      }
      const int ek = mk ? min(114, max(-100, max((int)(mk >> 23), (int)(mk >> 7 & 255) + 4) - (127 + 13))) : 0;
      const int ev = min(114, max(-60, max((int)(mv >> 23), (int)(mv >> 7 & 255) + 4) - (127 + 13)));
      const float fk = pow2f(-ek), fv = pow2f(-ev);
      const uint32_t kt = smem_u32(kbuf + st * C::KV_TILE), vt = smem_u32(vbuf + st * C::KV_TILE);
      const int row = un % H * PR_UN + 16 * dw + tr;
      ok = ok && mbar_wait_warp(&k_empty[st], ((it / S) & 1) ^ 1, tmo, abort_flag);
      if (!ok) break;
      if (lane == 0) {
        e_k[un % PR_E][dw] = pow2f(ek);
        e_v[un % PR_E][dw] = (float)ev;
        e_u[un % PR_E][dw] = fv;
      }
      // the next unit's parameters, and then its codes as registers come free, in flight meanwhile
      locate();
      params(kp0, un + PR_GROUPS, kn);
      params(vp0, un + PR_GROUPS, vn);
#pragma unroll
      for (int k = 0; k < 2; ++k) convert_row<NB, NG, BN>(kt, row + 8 * k, u, kw[k], kp[k], fk);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&k_full[st]);
      codes(kc0, kw);
      look_up(un + 2 * PR_GROUPS);
      ok = mbar_wait_warp(&v_empty[st], ((it / S) & 1) ^ 1, tmo, abort_flag);
      if (!ok) break;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // 16-bit units (2 u, j) and (2 u + 1, j), NB / 2 words apart and in the half that j says, make the word of
        // eight values; columns stay in the order 0 4 1 5 2 6 3 7 that nibbles come in, and the output puts them right
        uint32_t w[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j)
          w[j] = __byte_perm(vw[k][j >> 1], vw[k][NB / 2 + (j >> 1)], (j & 1) ? 0x7632 : 0x5410);
        convert_row<NB, NG, BN>(vt, row + 8 * k, u, w, vp[k], fv);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&v_full[st]);
      codes(vc0, vw);
      prefetch();
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          kp[k][i] = kn[k][i];
          vp[k][i] = vn[k][i];
        }
    }
    if (!ok && lane == 0 && !*abort_flag) fail();
  }

  // ------------------------------------------------------------------ MMA issuer
  if (warp >= C::MMA) setmaxnreg_dec<PrRegs<NQT>::MMA>();
  if (warp == C::MMA) {
    constexpr uint32_t idesc_s = idesc_f16_f32(128, BN);
    constexpr uint32_t idesc_o = idesc_f16_f32(128, D) | 1u << 16;  // B is MN-major
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_warp(bar, parity, tmo, abort_flag); };
    auto scores = [&](int q, int it) {
      if (!elect_one()) return;
      const uint32_t qa = tmem + C::Q_COL + (uint32_t)(q * (D / 2));
      const uint64_t qd = sdesc_k_sw128(smem_u32(smem + q * C::Q_TILE));
      const uint64_t kd = sdesc_k_sw128(smem_u32(kbuf + it % S * C::KV_TILE));
      const uint32_t d = tmem + (uint32_t)((q * NSB + it % NSB) * BN);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint64_t kk = kd + (k >> 2) * (BN * 128 / 16) + 2 * (k & 3);
        if (C::QT)
          mma_f16_ts(d, qa + 8 * k, kk, idesc_s, k > 0 ? 1u : 0u);
        else
          mma_f16(d, qd + (k >> 2) * (128 * 128 / 16) + 2 * (k & 3), kk, idesc_s, k > 0 ? 1u : 0u);
      }
      mma_commit(&s_full[q][it % NSB]);
      if (q == NQT - 1) mma_commit(&k_empty[it % S]);
    };
    bool ok = tmo != 0 && wait(&q_full, 0) && wait(&k_full[0], 0);
    tc_fence_after();
    if (ok)
      for (int q = 0; q < NQT; ++q) scores(q, 0);
    for (int it = 0; it < tiles && ok; ++it) {
      // the next scores: into the other buffer before this tile's products (its probabilities went into the
      // products before), or over this tile's once those are issued
      const bool more = it + 1 < tiles;
      if (NSB == 2 && more) {
        ok = wait(&k_full[(it + 1) % S], ((it + 1) / S) & 1);
        if (!ok) break;
        tc_fence_after();
        for (int q = 0; q < NQT; ++q) scores(q, it + 1);
      }
      ok = wait(&v_full[it % S], (it / S) & 1);
#pragma unroll
      for (int q = 0; q < NQT && ok; ++q) {
        const uint32_t o = tmem + C::O_COL + (uint32_t)(q * D);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const int un = it * H + h;
          ok = wait(&p_full[q][un & 1], (un >> 1) & 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t vd = sdesc_mn_sw128(smem_u32(vbuf + it % S * C::KV_TILE + h * PR_UN * 128), BN * 128);
            const uint32_t p = tmem + (uint32_t)((q * NSB + it % NSB) * BN + h * PR_UN);
#pragma unroll
            for (int k = 0; k < PR_UN / 16; ++k)
              mma_f16_ts(o, p + 8 * k, vd + k * (2048 / 16), idesc_o, un > 0 || k > 0 ? 1u : 0u);
            if constexpr (TWO) {
#pragma unroll
              for (int k = 0; k < PR_UN / 16; ++k) mma_f16_ts(o, p + 32 + 8 * k, vd + k * (2048 / 16), idesc_o, 1u);
            }
            mma_commit(&pv_done[q][un & 1]);
            if (q == NQT - 1 && h == H - 1) mma_commit(&v_empty[it % S]);
          }
        }
        if (NSB == 1 && ok && more) {
          if (q == 0) {
            ok = wait(&k_full[(it + 1) % S], ((it + 1) / S) & 1);
            tc_fence_after();
          }
          if (ok) scores(q, it + 1);
        }
      }
    }
    if (!ok && lane == 0 && !*abort_flag) fail();
    if (elect_one()) mma_commit(&drain_bar);
    mbar_wait_bounded(&drain_bar, 0, 1u << 20);
  }

  // ------------------------------------------------------------------ softmax
  if (warp < C::DEQ0) {
    setmaxnreg_inc<PrRegs<NQT>::SOFTMAX>();
    const int q = warp >> 2;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ot = tmem + lanes + C::O_COL + (uint32_t)(q * D);
    // queries: thread = row, scaled to fp16; what its softmax needs
    const int r = r0 + threadIdx.x;
    const bool live = r < a.rows;
    const int qi = live ? r / a.group : 0, h = live ? r - qi * a.group : 0;
    const int64_t base = (int64_t)b * a.qbs + (int64_t)qi * a.qts + ((int64_t)head * a.group + h) * D;
    float mx = 0.0f;
    if (live) {
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        float x[8];
        RawQ<false> raw;
        raw.load(a, base, c);
        raw.unpack(a, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = max_nan(mx, fabsf(x[i]));
      }
    }
    const int e = row_exponent(mx);
    const float up = row_scale(mx, e);
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[8];
        RawQ<false> raw;
        raw.zero();
        if (live) raw.load(a, base, 4 * c + i);
        raw.unpack(a, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[4 * i + k] = h2(x[2 * k] * up, x[2 * k + 1] * up);
        if (!C::QT)
          *reinterpret_cast<uint4*>(smem + q * C::Q_TILE + tile_off((int)threadIdx.x & 127, 4 * c + i, 128)) =
              make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
      if (C::QT) tmem_st16_u(tmem + lanes + C::Q_COL + (uint32_t)(q * (D / 2) + 16 * c), w);
    }
    if (C::QT)
      tmem_st_wait();
    else
      fence_proxy_async_smem();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&q_full);
    const float mul = fminf(pow2f(-e) * a.scale_log2, AT_TOP);
    int see_lo = 0, see_hi = 0;
    if (!live) {  // rows past the last: zero queries, masked nowhere but past the end
      see_hi = end;
    } else if (qi < nq) {
      see_hi = n;
      if (a.causal) {
        see_hi = n - nq + qi + 1;
        see_lo = after_window(a, see_hi);
      }
      see_hi = min(see_hi, end);
    }
    float yr = AT_M0, er = -60.0f, l = 0.0f;  // the reference: x and ev of the largest x + ev at its last move
    bool ok = true, big = false;
#pragma unroll 1
    for (int un = 0; un < units; ++un) {
      const int it = un / H;
      if (un % H == 0 && !mbar_wait_warp(&s_full[q][it % NSB], (it / NSB) & 1, tmo, abort_flag)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t stile = tmem + lanes + (uint32_t)((q * NSB + it % NSB) * BN + un % H * PR_UN);
      uint32_t x0[32], x1[32];
      tmem_ld32(stile, x0);
      tmem_ld32(stile + 32, x1);
      tmem_ld_wait_regs(x0);
      reg_fence(x1);
      const float4 ek4 = *reinterpret_cast<const float4*>(e_k[un % PR_E]);
      const float4 ev4 = *reinterpret_cast<const float4*>(e_v[un % PR_E]);
      // by 16 tokens; never 0, as masked scores are -inf
      float mk[4] = {fmaxf(mul * ek4.x, 1e-37f), fmaxf(mul * ek4.y, 1e-37f), fmaxf(mul * ek4.z, 1e-37f),
                     fmaxf(mul * ek4.w, 1e-37f)};
      float ev[4] = {ev4.x, ev4.y, ev4.z, ev4.w};
      const int t0 = lo + un * PR_UN;
      if (!__all_sync(FULL_MASK, t0 >= see_lo && t0 + PR_UN <= see_hi)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (t0 + i < see_lo || t0 + i >= see_hi) x0[i] = 0xff800000u;
          if (t0 + 32 + i < see_lo || t0 + 32 + i >= see_hi) x1[i] = 0xff800000u;
        }
      }
      float xt = AT_M0, top[4];  // the largest x + ev; the largest scores of each 16
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t(&x)[32] = i < 2 ? x0 : x1;
        float h0 = -INFINITY, h1 = -INFINITY;
#pragma unroll
        for (int k = 16 * (i & 1); k < 16 * (i & 1) + 16; k += 4) {
          h0 = fmaxf(h0, fmaxf(__uint_as_float(x[k]), __uint_as_float(x[k + 1])));
          h1 = fmaxf(h1, fmaxf(__uint_as_float(x[k + 2]), __uint_as_float(x[k + 3])));
        }
        top[i] = fmaxf(h0, h1);
        xt = fmaxf(xt, fmaf(top[i], mk[i], ev[i]));
      }
      // the products two units back are in (each phase is waited for in its turn: a later one could not be
      // told from it by parity)
      if (un > 1 && !mbar_wait_warp(&pv_done[q][un & 1], ((un >> 1) - 1) & 1, tmo, abort_flag)) {
        ok = false;
        break;
      }
      float less = yr + (er - 6.0f);  // what the probabilities' exponents leave off
      if (__builtin_expect(__any_sync(FULL_MASK, xt > less + 14.0f) || big, 0)) {
        float yn = yr, en = er;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = __fmul_rn(top[i], mk[i]);
          if (__fadd_rn(__fsub_rn(y, yn), ev[i] - en) > 0.0f) yn = y, en = ev[i];
        }
        const float by = __fadd_rn(__fsub_rn(yr, yn), er - en), f = ex2(by);
        l = l * ex2(0.5f * by) * ex2(0.5f * by);  // 2^-ev is in it: where 2^by alone is no more, it may be
        yr = yn;
        er = en;
        less = yr + (er - 6.0f);
        big = __any_sync(FULL_MASK, (fabsf(yr) > 4096.0f && yr != AT_M0) || er > 20.0f);
        if (un > 0 && __any_sync(FULL_MASK, f != 1.0f)) {  // once the products so far are in
          if (!mbar_wait_warp(&pv_done[q][(un - 1) & 1], ((un - 1) >> 1) & 1, tmo, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t v[16];
            float w[16];
            tmem_ld16(ot + c, v);
            tmem_ld_wait_regs16(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __uint_as_float(v[i]) * f;
            tmem_st16(ot + c, w);
          }
        }
      }
      if (__builtin_expect(big, 0)) {
        // values far below the reference's, zeros among them, add nothing but still weigh: with an ev that leaves p above 2^-126
#pragma unroll
        for (int i = 0; i < 4; ++i) ev[i] = fmaxf(ev[i], er - 100.0f);
      }
      if (D < 256 && __builtin_expect(big, 0)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          x0[i] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(x0[i]), mk[i >> 4]), yr));
          x1[i] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(x1[i]), mk[2 + (i >> 4)]), yr));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) mk[i] = 1.0f;
        less = er - 6.0f;
      }
      float sum[4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t(&x)[32] = half ? x1 : x0;
        uint32_t p[16];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // m x + off; with 256 values always m x - yr by itself first, as dequantization leaves the time for it and a branch
          // (`big`) made the compiler spill (36 rows: 42 us, with the branch 45)
          const float m = mk[2 * half + j], off = ev[2 * half + j] - less;
          const float last = D < 256 ? 0.0f : ev[2 * half + j] - er + 6.0f;
          const uint64_t m2 = pack_f2(m, m), off2 = pack_f2(off, off), last2 = pack_f2(last, last);
          uint64_t s2 = 0;
#pragma unroll
          for (int i = 8 * j; i < 8 * j + 8; ++i) {
            float a0, a1;
            if constexpr (D < 256) {
              unpack_f2(fma_f2(pack_f2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), m2, off2), a0, a1);
            } else {  // (the packed product and difference would become one multiply-add again)
              a0 = __fsub_rn(__fmul_rn(__uint_as_float(x[2 * i]), m), yr);
              a1 = __fsub_rn(__fmul_rn(__uint_as_float(x[2 * i + 1]), m), yr);
              unpack_f2(add_f2(pack_f2(a0, a1), last2), a0, a1);
            }
            a0 = ex2(a0);
            a1 = ex2(a1);
            s2 = add_f2(s2, pack_f2(a0, a1));
            p[i] = h2(a0, a1);
            if constexpr (TWO) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p[i]));
              x[2 * i] = h2(a0 - f.x, a1 - f.y);
            }
          }
          float s0, s1;
          unpack_f2(s2, s0, s1);
          sum[2 * half + j] = s0 + s1;
        }
        tmem_st16_u(stile + 16 * half, p);
        if constexpr (TWO) {
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] = x[2 * i];
          tmem_st16_u(stile + 32 + 16 * half, p);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) l = fmaf(sum[i], __builtin_expect(big, 0) ? ex2(-ev[i]) : e_u[un % PR_E][i], l);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[q][un & 1]);
    }
    for (int un = units > 1 ? units - 2 : 0; un < units && ok; ++un)
      ok = mbar_wait_warp(&pv_done[q][un & 1], (un >> 1) & 1, tmo, abort_flag);
    if (!ok && lane == 0 && !*abort_flag) fail();
    if (ok) {
      tc_fence_after();
      const int64_t orow = out_row(a, b, head, r < a.rows ? r : 0);
      const bool whole = a.chunks == 1;
      // partial sums leave without their 2^(6 - er); a row that sees nothing: 0; NaN stays
      const float inv = !whole ? pow2f((int)er - 6) : (l > 0.0f ? 1.0f / l : l);
      float* part = whole ? nullptr : a.part + (orow * a.chunks + ch) * D;
      if (!whole && r < a.rows) {
        a.stats[(orow * a.chunks + ch) * 2] = yr;
        a.stats[(orow * a.chunks + ch) * 2 + 1] = l * inv;
      }
#pragma unroll 1
      for (int c = 0; c < D; c += 16) {
        uint32_t v[16];
        tmem_ld16(ot + c, v);
        tmem_ld_wait_regs16(v);
        float w[2][8];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i >> 3][(i & 7) >> 1 | (i & 1) << 2] = __uint_as_float(v[i]) * inv;  // 0 4 1 5 2 6 3 7
        if (r < a.rows) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!whole)
              store8(part + c + 8 * i, w[i]);
            else if (a.type == FGQ_BF16)
              store8(static_cast<__nv_bfloat16*>(a.out) + orow * D + c + 8 * i, w[i]);
            else
              store8(static_cast<__half*>(a.out) + orow * D + c + 8 * i, w[i]);
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == C::MMA) {
    tc_fence_after();
    tmem_dealloc(tmem, C::COLS);
  }
}

template <int D, int G, int NQT, bool TWO>
fgq_status launch_prompt_as(const AttnArgs& a, unsigned blocks, cudaStream_t s) {
  using C = PrCfg<D, NQT>;
  static_assert(C::SMEM + 2048 <= 232448, "shared memory budget");
  static_assert(C::Q_COL <= 512, "tensor memory budget");
  if (!tc::smem_attr_once<kv_prompt_kernel<D, G, NQT, TWO>>(C::SMEM)) return FGQ_ERR_CUDA;
  kv_prompt_kernel<D, G, NQT, TWO><<<blocks, C::THREADS, C::SMEM, s>>>(a);
  return after_launch();
}

template <int D, int G, int NQT>
fgq_status launch_prompt(const AttnArgs& a, unsigned blocks, cudaStream_t s) {
  return a.type == FGQ_F16 ? launch_prompt_as<D, G, NQT, true>(a, blocks, s) : launch_prompt_as<D, G, NQT, false>(a, blocks, s);
}

template <int D, int G>
AttnKernel pick_prompt(int rows) {
  if constexpr (D <= 128) {
    if (rows > 128) return {launch_prompt<D, G, 2>, 256, 1, false, 9.0f, 9.0f, D == 64 ? 73.0f : 54.0f};
  }
  return {launch_prompt<D, G, 1>, 128, 1, false, 8.0f, 8.0f, D == 64 ? 122.0f : (D == 128 ? 93.0f : 47.0f)};
}

}  // namespace

namespace dec {

AttnKernel prompt_kernel(int D, int G, int rows) {
  if (D == 64) return G == 32 ? pick_prompt<64, 32>(rows) : pick_prompt<64, 64>(rows);
  if (D == 128)
    return G == 32 ? pick_prompt<128, 32>(rows) : G == 64 ? pick_prompt<128, 64>(rows) : pick_prompt<128, 128>(rows);
  return G == 32 ? pick_prompt<256, 32>(rows) : G == 64 ? pick_prompt<256, 64>(rows) : pick_prompt<256, 128>(rows);
}

}  // namespace dec
}  // namespace fgq
