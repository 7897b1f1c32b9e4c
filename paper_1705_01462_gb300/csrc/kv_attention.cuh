// Attention over the 4-bit cache, few query rows: the cache is read once, in chunks of tokens that
// blocks take side by side, and dequantized on the way into the matrix instructions.
//
// Mathematics.  With k = lo + s c, the score of token t and query row n is
//   scale * sum_g ( s_tg (q_ng . c_tg) + lo_tg sum(q_ng) )         (g: groups of the head's values)
// and with v likewise, the output's value d in group g is
//   sum_t (p_nt s_tg) (c_td - 8) + sum_t p_nt (lo_tg + 8 s_tg),
// so both products run on the codes themselves and the parameters are applied to scores and to
// probabilities.  A code in the low bits of an fp16 is the subnormal c 2^-24 (or 16 c 2^-24, four bits
// up): one AND and one packed product per two codes make the matrix operand c 2^-9, exactly.  (The
// subnormals themselves lose up to ten bits in the instructions' sums: 7e-5 of the output instead of
// 1e-6 for fp32.)  Tokens (keys) and values' dimensions (V)
// are the M = 16 rows of mma.m16n8k16, eight query rows its columns, so that a group of eight query
// heads pads nothing.  These legacy matrix instructions do here: 16 of them per 2 KB of cache leave the
// tensor pipe a third busy at full HBM rate, and tcgen05 would want the dequantized operands in shared
// or tensor memory first.
//
// What is rounded: queries to fp16 after scaling each row by a power of two (exact for bf16 and fp16;
// fp32 queries take two fp16 parts, SPLIT), and p s to fp16 (two parts for SPLIT; value codes are centred
// so that its error meets values of the size of v).  For bf16 outputs that adds 1% to the output's own rounding, for fp16
// ones a third (2.7e-4 of the output against 2.1e-4, single tokens over 4000; 3.4e-4 at most among 1000 cases): a second part would double the products with
// the values (in kv_prompt.cu, where it was taken, that is a fifth of the time).  Scores, statistics and sums are fp32; the instructions cut
// their sums off, so SPLIT adds each step's products to the output rounded (51 x 42000 tokens: 1.1e-5 of the
// output to 6e-7, 207 to 222 us), which would not show in 16-bit outputs.
//
// Softmax.  Probabilities are held as 2^(mul (x - r) + 6 - log2(sigma)): x is a score before its scaling, mul the row's factor
// to log2 units, r the row's largest x at its last move, and sigma a power of two at or above every value scale met, so that
// p s fits fp16 whatever the values' magnitude.  r moves only when a score exceeds it by more than 8 / mul, or a value
// scale sigma: the common tile needs one vote instead of a reduction per row.  The difference comes before the product, as
// mul x - mul r in one multiply-add is off by the rounding of mul r, which scores past 2^25 turn into infinities or zeros.  Sums
// leave a warp without their 2^(6 - log2(sigma)), so that a join meets no factor but the scores'.
//
// Split.  A block of 4 warps takes `chunk` tokens of one (sequence, kv head, tile of 8 NT query rows);
// each warp streams every fourth tile through a ring of bulk copies of its own (no barrier
// between warps), and the warps' sums are joined in shared memory.  Up to eight chunks of one wave are a
// cluster, which joins through shared memory too; more leave (r, l, sum) in fp32, which a second kernel joins.
//
// What bounds it.  One token each of 16 sequences of 16384 tokens, 32 query and 8 kv heads of 128 values, groups of 64: 80 us
// for 302 MB, 56% of the copy rate, with no unit saturated: ALU pipe 52%, tensor pipe 19%, issue slots 60%, DRAM 52% busy
// over the launch.  Twelve warps an SM do not fill one another's waits.  More or fewer blocks an SM, shorter tiles, e4m3
// products and codes with an offset in place of the packed product were all slower.  One sequence of 131071 tokens, 64 query
// heads, groups of 128: 41 us (143 MB).
#pragma once

#include "decoder_internal.cuh"
#include "ptx_sm100.cuh"

namespace fgq {
namespace dec {

struct AttnArgs {
  CacheView c;
  const void* q;
  void* out;
  int64_t qbs, qts;  // q's batch and token strides, elements
  const int32_t* seq_lens;
  const int32_t* q_lens;
  float* part;   // [row][chunks] partial sums of D values each, or nullptr (one chunk)
  float* stats;  // [row][chunks][2]: r, l
  unsigned int* err;
  uint64_t timeout_ns;
  float scale_log2;  // scale * log2(e)
  int type, B, T, q_heads, group, rows, row_tiles, chunks, chunk, causal, window;
  int cluster;  // the chunks of a tile are a cluster and join in shared memory
};

constexpr int AT_WARPS = 4;
constexpr int AT_STEP = 32;  // tokens a warp computes at a time
constexpr float AT_M0 = -3.4e38f;   // reference of a row that has seen nothing
constexpr float AT_TOP = 3.39e38f;  // largest magnitude of the others, in log2 units
constexpr float AT_EMPTY = -INFINITY;  // in place of a reference: a cluster's chunk without work, whose sums were never written

// Shared memory of one ring stage: TILE rows of key codes, value codes, key and value parameters.  Tiles of 64
// tokens where they fit: bulk copies are the fewer and the larger for it (524 k copies of 1 KB and 128 bytes
// took as long as 300 MB from HBM).
template <int NB, int GB>
struct AttnSmem {
  static constexpr int D = 32 * NB, NG = NB / GB;
  static constexpr int TILE = NB == 8 ? 32 : 64, STAGES = NB == 2 ? 3 : 2;
  static constexpr int ROW = D / 2, PAR = 4 * NG;
  static constexpr int STAGE = TILE * 2 * (ROW + PAR);
  static constexpr int RING = AT_WARPS * STAGES * STAGE;
  static constexpr int BARS = AT_WARPS * STAGES * 8;
  template <int NT>
  static constexpr int bytes() {
    // the warps' sums reuse the ring
    const int join = AT_WARPS * 8 * NT * (D + 2) * 4;
    return (RING > join ? RING : join) + BARS + 16;
  }
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// c 2^-9 for the two codes in the low nibbles of w's halves, or the next ones: subnormals scaled to normal
// fp16, exactly.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w & 0x000f000fu), "r"(0x78007800u));  // 2^15
  return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w & 0x00f000f0u), "r"(0x68006800u));  // 2^11
  return r;
}
// (c - 8) 2^-9 likewise.
__device__ __forceinline__ uint32_t centred_lo(uint32_t w) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w & 0x000f000fu), "r"(0x78007800u), "r"(0xa400a400u));  // -2^-6
  return r;
}
__device__ __forceinline__ uint32_t centred_hi(uint32_t w) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w & 0x00f000f0u), "r"(0x68006800u), "r"(0xa400a400u));
  return r;
}
__device__ __forceinline__ uint32_t h2(float a, float b) { return pack2(a, b, __half()); }
__device__ __forceinline__ float2 f2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// The words of one thread's piece of a cache row in shared memory (4 N bytes, aligned as that).
template <int N>
__device__ __forceinline__ void lds_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  }
}

// Eight query elements 8 e .. 8 e + 7 from element `base` on, as loaded (F32: 32 bytes, else 16) and as fp32.
template <bool F32>
struct RawQ {
  uint4 v[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const AttnArgs& a, int64_t base, int e) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.q) + (base + 8 * e) * (F32 ? 4 : 2));
    v[0] = __ldg(p);
    if (F32) v[F32 ? 1 : 0] = __ldg(p + 1);
  }
  __device__ __forceinline__ void zero() { v[0] = v[F32 ? 1 : 0] = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void unpack(const AttnArgs& a, float (&x)[8]) const {
    if constexpr (F32) {
      const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else if (a.type == FGQ_BF16) {
      unpack8(v[0], x, __nv_bfloat16());
    } else {
      unpack8(v[0], x, __half());
    }
  }
};

__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t at, float v) {
  if (a.type == FGQ_F32)
    static_cast<float*>(a.out)[at] = v;
  else if (a.type == FGQ_BF16)
    static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(a.out)[at] = __float2half_rn(v);
}

// Exponent e of the power of two that takes a query row's largest magnitude mx to [2^13, 2^14) (below it for subnormal ones).
__device__ __forceinline__ int row_exponent(float mx) {
  return mx > 0.0f ? max(-114, min(126, 13 + 127 - (int)((__float_as_uint(mx) >> 23) & 255))) : 0;
}
// What the elements of a query row with largest magnitude mx are multiplied by, 2^e; NaN for a row that holds Inf or NaN: no
// softmax of its scores is defined, and scores of one infinity would pass for a row that sees nothing.
__device__ __forceinline__ float row_scale(float mx, int e) { return nonfinite(mx) ? __uint_as_float(0x7fc00000u) : pow2f(e); }

// Tokens of sequence b: at most what the table can hold (more is an error), less than 2^31 - 2^12.
__device__ __forceinline__ int seq_len(const AttnArgs& a, int b) {
  const int n = __ldg(a.seq_lens + b);
  const int most = (int)min((int64_t)a.c.max_pages * a.c.page_size, (int64_t)INT32_MAX - 4096);
  if (n > most) record_error(a.err, FGQ_ERR_ARG);
  return min(n, most);
}

// First position that a window ending before position `end` leaves (no difference that could wrap around).
__device__ __forceinline__ int after_window(const AttnArgs& a, int end) { return a.window && end > a.window ? end - a.window : 0; }

// First and one past the last position that any of the query rows [i0, i1] (by query index) of a
// sequence of n tokens and nq queries sees.
__device__ __forceinline__ void visible(const AttnArgs& a, int n, int nq, int i0, int i1, int& first, int& end) {
  i1 = min(i1, nq - 1);
  if (i1 < i0 || n <= 0) {
    first = end = 0;
    return;
  }
  if (!a.causal) {
    first = 0;
    end = n;
    return;
  }
  end = max(n - nq + i1 + 1, 0);
  first = after_window(a, n - nq + i0 + 1);
  if (end <= first) first = end = 0;
}

// A row of the output; its value from a sum and a denominator (a row that saw nothing: 0; NaN stays).
__device__ __forceinline__ int64_t out_row(const AttnArgs& a, int b, int head, int r) {
  const int qi = r / a.group, h = r - qi * a.group;
  return ((int64_t)b * a.T + qi) * a.q_heads + (int64_t)head * a.group + h;
}
__device__ __forceinline__ float normalise(float v, float l) { return l > 0.0f ? v / l : (l == 0.0f ? 0.0f : l); }

// A float at this block's shared address `p`, in the cluster's block `rank`.
__device__ __forceinline__ float ld_cluster(const float* p, uint32_t rank) {
  uint32_t at;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// The rows of a cluster's blocks (chunks of one tile of rows), each block's sums at jo [row][D] and its r, l
// at js [row][2], joined and stored: block `rank` takes every a.chunks-th run of 128 values.
template <int NB, int NR>
__device__ __forceinline__ void join_cluster(const AttnArgs& a, int b, int head, int r0, const float* jo,
                                             const float* js, int rank) {
  constexpr int D = 32 * NB;
  for (int i = threadIdx.x + 32 * AT_WARPS * rank; i < NR * D; i += 32 * AT_WARPS * a.chunks) {
    const int row = i / D, d = i % D, r = r0 + row;
    if (r >= a.rows) break;
    float m[8], mm = AT_M0, ll = 0.0f, v = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      m[c] = c < a.chunks ? ld_cluster(js + 2 * row, c) : AT_EMPTY;
      mm = fmaxf(mm, m[c]);
    }
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (m[c] != AT_EMPTY) {
        const float f = ex2(m[c] - mm);
        ll = fmaf(f, ld_cluster(js + 2 * row + 1, c), ll);
        v = fmaf(f, ld_cluster(jo + row * D + d, c), v);
      }
    store_out(a, out_row(a, b, head, r) * D + d, normalise(v, ll));
  }
}

// Blocks of one SM, by registers and shared memory.  Two tiles of rows of 128 values need 229 to 255 registers: held to the 168 of
// three blocks they spilled 236 to 692 bytes (16 rows, 32 sequences of 2000 tokens: 51 us, and 33 with two blocks).
template <int NB, int NT>
constexpr int attention_blocks_per_sm() {
  return NB == 8 || (NB == 4 && NT == 2) ? 2 : 3;
}

template <int NB, int GB, bool SPLIT, int NT>
__global__ void __launch_bounds__(32 * AT_WARPS, attention_blocks_per_sm<NB, NT>())
    kv_attention_kernel(const __grid_constant__ AttnArgs a) {
  using S = AttnSmem<NB, GB>;
  constexpr int D = S::D, NG = S::NG, ROW = S::ROW, PAR = S::PAR, STAGES = S::STAGES, TILE = S::TILE;
  constexpr int NQ = SPLIT ? 2 : 1;  // fp16 parts of a query and of a probability
  constexpr int NR = 8 * NT;         // query rows of the block
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int BODY = S::template bytes<NT>() - S::BARS - 16;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + BODY);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + BODY + S::BARS);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;

  // block -> (sequence, kv head, tile of query rows, chunk); a cluster is the chunks of one tile
  int id = blockIdx.x;
  const int ch = id % a.chunks;
  id /= a.chunks;
  const int rt = id % a.row_tiles;
  id /= a.row_tiles;
  const int head = id % a.c.kv_heads;
  const int b = id / a.c.kv_heads;
  const int r0 = rt * NR;

  // the queries are on their way before the cache is: behind its first tiles they took four microseconds
  RawQ<SPLIT> qraw[NT][NB];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = r0 + 8 * nt + g, qi = r / a.group;
    const int64_t base = (int64_t)b * a.qbs + (int64_t)qi * a.qts + ((int64_t)head * a.group + (r - qi * a.group)) * D;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      qraw[nt][j].zero();
      if (r < a.rows) qraw[nt][j].load(a, base, 4 * j + t);
    }
  }

  const int n = seq_len(a, b);
  const int nq = a.q_lens ? min(__ldg(a.q_lens + b), a.T) : a.T;
  int first, end;
  visible(a, n, nq, r0 / a.group, (min(r0 + NR, a.rows) - 1) / a.group, first, end);
  const int seen = first;  // tokens before it share its block of 16 and may never have been written
  first &= ~15;
  // this block's tokens [lo, hi): chunks start a multiple of 32 after `first`; the last one takes the rest
  const int64_t lo64 = (int64_t)first + (int64_t)ch * a.chunk;
  const int lo = lo64 < end ? (int)lo64 : end;
  const int hi = ch == a.chunks - 1 ? end : (int)min((int64_t)end, lo64 + a.chunk);

  float* jo = reinterpret_cast<float*>(smem);  // [warp][row][D]: the warps' sums, over the ring
  float* js = jo + AT_WARPS * NR * D;          // [warp][row][2]: r, l
  if (lo >= hi) {  // nothing here: zero output where there is one chunk only, else the join skips it
    if (a.cluster) {
      if (threadIdx.x < NR) js[2 * threadIdx.x] = AT_EMPTY;
      cluster_sync();
      join_cluster<NB, NR>(a, b, head, r0, jo, js, ch);
      cluster_sync();
    } else if (a.chunks == 1) {
      for (int i = threadIdx.x; i < NR * D; i += 32 * AT_WARPS) {
        const int r = r0 + i / D;
        if (r < a.rows) {
          const int qi = r / a.group, h = r - qi * a.group;
          store_out(a, (((int64_t)b * a.T + qi) * a.q_heads + (int64_t)head * a.group + h) * D + i % D, 0.0f);
        }
      }
    }
    return;
  }

  pdl_trigger();  // the join may be brought up; it waits for this kernel's end
  if (threadIdx.x == 0) {
    for (int i = 0; i < AT_WARPS * STAGES; ++i) mbar_init(&bars[i], 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();

  uint8_t* ring = smem + warp * STAGES * S::STAGE;
  uint64_t* bar = bars + warp * STAGES;
  const int tiles_all = (hi - lo + TILE - 1) / TILE;
  const int tiles = (tiles_all - warp + AT_WARPS - 1) / AT_WARPS;  // this warp's

  // lanes 4 k + array copy (key codes, value codes, key, value parameters) from 16-token block k of the tile on,
  // where that is the tile's first or its page's: as many blocks as lie in the page
  constexpr int BLOCKS = TILE / 16;
  const bool par = lane & 2, val = lane & 1;
  const int blk = lane >> 2;
  const uint32_t row_bytes = par ? PAR : ROW;
  const uint8_t* src = par ? reinterpret_cast<const uint8_t*>(val ? a.c.v_params : a.c.k_params)
                           : (val ? a.c.v_codes : a.c.k_codes);
  const uint32_t dst = smem_u32(ring) + (par ? 2 * TILE * ROW + (val ? TILE * PAR : 0) : (val ? TILE * ROW : 0)) +
                       blk * 16 * row_bytes;
  const int32_t* table = a.c.table + (int64_t)b * a.c.max_pages;
  int ptok = lo + warp * TILE + 16 * blk;  // this lane's block of the next tile to look up
  int page = -1, slot = 0, run = 0;        // of the next tile to issue: page, slot, tokens to copy
  auto look_up = [&]() {  // positions below hi are inside the table: seq_len() sees to it
    run = 0;
    if (blk < BLOCKS && ptok < hi) {
      const uint32_t pi = page_of(a.c, (uint32_t)ptok);
      slot = ptok - (int)pi * a.c.page_size;
      if (blk == 0 || slot == 0) {
        page = __ldg(table + pi);
        run = min(min(TILE - 16 * blk, a.c.page_size - slot), (hi - ptok + 15) & ~15);
      }
    }
    ptok += AT_WARPS * TILE;
  };
  int ist = 0;  // stage of the next tile to issue
  auto issue = [&]() {
    if (run > 0 && (page < 0 || page >= a.c.pages)) {
      record_error(a.err, FGQ_ERR_ARG);
      run = 0;
    }
    const uint32_t tokens = __reduce_add_sync(FULL_MASK, (lane & 3) == 0 ? (uint32_t)run : 0u);
    if (lane == 0) mbar_arrive_expect_tx(&bar[ist], tokens * 2u * (ROW + PAR));
    __syncwarp();
    if (run > 0)
      bulk_load(dst + ist * S::STAGE, src + (((int64_t)page * a.c.kv_heads + head) * a.c.page_size + slot) * row_bytes,
                (uint32_t)run * row_bytes, &bar[ist]);
    ist = ist + 1 == STAGES ? 0 : ist + 1;
  };
  look_up();
  int issued = 0;
#pragma unroll 1
  for (; issued < STAGES && issued < tiles; ++issued) {
    issue();
    look_up();
  }

  // queries as operand columns: this thread's part of row 8 nt + g, and what rows 8 nt + 2 t, + 1 need
  uint32_t qf[NT][NQ][2 * NB][2];
  float qsum[NT][NG][2], mul[NT][2];
  int see_lo[NT][2], see_hi[NT][2];  // tokens [see_lo, see_hi) that rows 8 nt + 2 t, + 1 see
  int all_lo = 0, all_hi = INT32_MAX;  // tokens that every row sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = r0 + 8 * nt + g;
    const bool live = r < a.rows;
    const int qi = live ? r / a.group : 0;
    float x[NB][8];
    float mx = 0.0f;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      qraw[nt][j].unpack(a, x[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = max_nan(mx, fabsf(x[j][i]));
    }
    mx = max_nan(mx, __shfl_xor_sync(FULL_MASK, mx, 1));
    mx = max_nan(mx, __shfl_xor_sync(FULL_MASK, mx, 2));
    const int e = row_exponent(mx);
    const float up = row_scale(mx, e);
    float sums[NG];
#pragma unroll
    for (int i = 0; i < NG; ++i) sums[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {  // pairs (0, 1), (2, 3), ..
        const float p0 = x[j][2 * w] * up, p1 = x[j][2 * w + 1] * up;
        const uint32_t hw = h2(p0, p1);
        const float2 back = f2(hw);
        float s0 = back.x, s1 = back.y;
        qf[nt][0][2 * j + (w >> 1)][w & 1] = hw;
        if constexpr (SPLIT) {
          const uint32_t lw = h2(p0 - back.x, p1 - back.y);
          qf[nt][NQ - 1][2 * j + (w >> 1)][w & 1] = lw;
          const float2 rest = f2(lw);
          s0 += rest.x, s1 += rest.y;
        }
        sums[j / GB] += s0 + s1;
      }
    }
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      sums[i] += __shfl_xor_sync(FULL_MASK, sums[i], 1);
      sums[i] += __shfl_xor_sync(FULL_MASK, sums[i], 2);
      sums[i] *= 0.001953125f;  // 2^-9: the codes' scale
    }
    const float m = fminf(fmaxf(pow2f(-e) * a.scale_log2 * 512.0f, 1e-37f), AT_TOP);  // finite: 0 m is 0
    // positions of the row: [sl, sh)
    int sl = 0, sh = live ? 0 : INT32_MAX;  // rows past the last: zero queries, masked nowhere
    if (live && qi < nq) {
      sh = n, sl = 0;
      if (a.causal) {
        sh = n - nq + qi + 1;
        sl = after_window(a, sh);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int from = 4 * (2 * t + u);
#pragma unroll
      for (int i = 0; i < NG; ++i) qsum[nt][i][u] = __shfl_sync(FULL_MASK, sums[i], from);
      mul[nt][u] = __shfl_sync(FULL_MASK, m, from);
      see_lo[nt][u] = __shfl_sync(FULL_MASK, sl, from);
      see_hi[nt][u] = min(__shfl_sync(FULL_MASK, sh, from), end);
      all_lo = max(all_lo, see_lo[nt][u]);
      all_hi = min(all_hi, see_hi[nt][u]);
    }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    all_lo = max(all_lo, __shfl_xor_sync(FULL_MASK, all_lo, o));
    all_hi = min(all_hi, __shfl_xor_sync(FULL_MASK, all_hi, o));
  }

  // sums of 2^(mul (x - r) + off) times codes, times lo, and alone; a row's -r, which moves when a score passes its limit
  float o[NT][NB][2][4], olo[NT][NG][2], l[NT][2], nref[NT][2], limit[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      nref[nt][u] = -AT_M0;
      limit[nt][u] = -INFINITY;
      l[nt][u] = 0.0f;
#pragma unroll
      for (int i = 0; i < NG; ++i) olo[nt][i][u] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][j][u][i] = 0.0f;
  }
  // a power of two at or above every value scale met so far, 2^-60 at least; 0 before the first scale above 0: groups of equal
  // values, zeros among them, have none, and p with 2^60 in it would take them past fp32's range or out of a join
  float sigma = 0.0f;
  float off = 6.0f;  // 6 - log2(sigma), or 6

  bool ok = true;
  int done = 0, tile0 = lo + warp * TILE, st = 0;
  uint32_t phase = 0;
#pragma unroll 1
  for (; done < tiles; ++done, tile0 += AT_WARPS * TILE) {
    // a limit of 0 (a test's) expires at once, whether the copy has landed or not
    if (a.timeout_ns == 0 || !mbar_wait_warp(&bar[st], phase, a.timeout_ns, abort_flag)) {
      ok = false;
      break;
    }
#pragma unroll 1
    for (int step = 0; step < TILE; step += AT_STEP) {
      const int tok0 = tile0 + step;
      if (TILE > AT_STEP && tok0 >= hi) break;
      const uint8_t* kc = ring + st * S::STAGE + step * ROW;
      const uint8_t* vc = kc + TILE * ROW;
      const uint32_t* kp = reinterpret_cast<const uint32_t*>(ring + st * S::STAGE + 2 * TILE * ROW) + step * NG;
      const uint32_t* vp = kp + TILE * NG;

      // scores of tokens 16 mt + g, + 8 for rows 8 nt + 2 t, + 1
      float x[2][NT][4];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint32_t wa[NB], wb[NB];
        lds_words<NB>(kc + (16 * mt + g) * ROW + t * 4 * NB, wa);
        lds_words<NB>(kc + (16 * mt + g + 8) * ROW + t * 4 * NB, wb);
        uint32_t pa[NG], pb[NG];
        lds_words<NG>(reinterpret_cast<const uint8_t*>(kp + (16 * mt + g) * NG), pa);
        lds_words<NG>(reinterpret_cast<const uint8_t*>(kp + (16 * mt + g + 8) * NG), pb);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[mt][nt][i] = 0.0f;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          float acc[NT][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nt][i] = 0.0f;
#pragma unroll
          for (int jj = 0; jj < GB; ++jj) {
            const int j = gi * GB + jj;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t va = u ? wa[j] >> 8 : wa[j], vb = u ? wb[j] >> 8 : wb[j];
              const uint32_t a0 = codes_lo(va), a1 = codes_lo(vb), a2 = codes_hi(va), a3 = codes_hi(vb);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int p = 0; p < NQ; ++p)
                  mma16816(acc[nt], a0, a1, a2, a3, qf[nt][p][2 * j + u][0], qf[nt][p][2 * j + u][1]);
            }
          }
          const float sa = __uint_as_float(pa[gi] << 16), la = __uint_as_float(pa[gi] & 0xffff0000u);
          const float sb = __uint_as_float(pb[gi] << 16), lb = __uint_as_float(pb[gi] & 0xffff0000u);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            x[mt][nt][0] = fmaf(la, qsum[nt][gi][0], fmaf(sa, acc[nt][0], x[mt][nt][0]));
            x[mt][nt][1] = fmaf(la, qsum[nt][gi][1], fmaf(sa, acc[nt][1], x[mt][nt][1]));
            x[mt][nt][2] = fmaf(lb, qsum[nt][gi][0], fmaf(sb, acc[nt][2], x[mt][nt][2]));
            x[mt][nt][3] = fmaf(lb, qsum[nt][gi][1], fmaf(sb, acc[nt][3], x[mt][nt][3]));
          }
        }
      }
      const bool whole = tok0 >= all_lo && tok0 + AT_STEP <= all_hi;
      if (!whole) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = tok0 + 16 * mt + g + 8 * (i >> 1);
              if (tok < see_lo[nt][i & 1] || tok >= see_hi[nt][i & 1]) x[mt][nt][i] = -INFINITY;
            }
      }

      // value parameters of this thread's four tokens; tokens past the end, or before the first one seen, hold nothing
      uint32_t vw[2][2][NG];
      float smax = 0.0f;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          lds_words<NG>(reinterpret_cast<const uint8_t*>(vp + (16 * mt + g + 8 * u) * NG), vw[mt][u]);
          if (!whole && (tok0 + 16 * mt + g + 8 * u >= hi || tok0 + 16 * mt + g + 8 * u < seen))
#pragma unroll
            for (int i = 0; i < NG; ++i) vw[mt][u][i] = 0u;
#pragma unroll
          for (int i = 0; i < NG; ++i) smax = fmaxf(smax, __uint_as_float(vw[mt][u][i] << 16));
        }

      bool move = smax > sigma;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          move |= fmaxf(fmaxf(x[0][nt][u], x[0][nt][2 + u]), fmaxf(x[1][nt][u], x[1][nt][2 + u])) > limit[nt][u];
      if (__any_sync(FULL_MASK, move)) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) smax = fmaxf(smax, __shfl_xor_sync(FULL_MASK, smax, s));
        if (smax > sigma)  // the next power of two
          sigma = fmaxf(__uint_as_float((__float_as_uint(smax) + 0x7fffffu) & 0x7f800000u), 8.6736174e-19f);
        const float now = sigma > 0.0f ? 6.0f - (float)((int)(__float_as_uint(sigma) >> 23) - 127) : 6.0f, by = now - off;
        off = now;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float h = fmaxf(fmaxf(x[0][nt][u], x[0][nt][2 + u]), fmaxf(x[1][nt][u], x[1][nt][2 + u]));
#pragma unroll
            for (int s = 16; s >= 4; s >>= 1) h = fmaxf(h, __shfl_xor_sync(FULL_MASK, h, s));
            const float nr = fminf(nref[nt][u], -h), f = ex2(fmaf(nr - nref[nt][u], mul[nt][u], by));
            nref[nt][u] = nr;
            if (h > -INFINITY) limit[nt][u] = __fadd_rd(8.0f / mul[nt][u], -nr);
            l[nt][u] *= f;
#pragma unroll
            for (int i = 0; i < NG; ++i) olo[nt][i][u] *= f;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                o[nt][j][w][u] *= f;
                o[nt][j][w][2 + u] *= f;
              }
          }
      }

#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint32_t pf[NT][NG][NQ][2];  // probabilities times value scales as operand columns
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
          const uint64_t nr2 = pack_f2(nref[nt][0], nref[nt][1]), m2 = pack_f2(mul[nt][0], mul[nt][1]), off2 = pack_f2(off, off);
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            unpack_f2(fma_f2(add_f2(pack_f2(x[mt][nt][i], x[mt][nt][i + 1]), nr2), m2, off2), p[i], p[i + 1]);
            p[i] = ex2(p[i]);
            p[i + 1] = ex2(p[i + 1]);
          }
          l[nt][0] += p[0] + p[2];
          l[nt][1] += p[1] + p[3];
#pragma unroll
          for (int gi = 0; gi < NG; ++gi) {
            const float sa = __uint_as_float(vw[mt][0][gi] << 16), sb = __uint_as_float(vw[mt][1][gi] << 16);
            const float la = fmaf(8.0f, sa, __uint_as_float(vw[mt][0][gi] & 0xffff0000u));  // the codes' centre
            const float lb = fmaf(8.0f, sb, __uint_as_float(vw[mt][1][gi] & 0xffff0000u));
            olo[nt][gi][0] = fmaf(p[0], la, fmaf(p[2], lb, olo[nt][gi][0]));
            olo[nt][gi][1] = fmaf(p[1], la, fmaf(p[3], lb, olo[nt][gi][1]));
            const float w0 = p[0] * sa, w1 = p[1] * sa, w2 = p[2] * sb, w3 = p[3] * sb;
            const uint32_t ha = h2(w0, w1), hb = h2(w2, w3);
            pf[nt][gi][0][0] = movmatrix(ha);
            pf[nt][gi][0][1] = movmatrix(hb);
            if constexpr (SPLIT) {
              const float2 ra = f2(ha), rb = f2(hb);
              pf[nt][gi][NQ - 1][0] = movmatrix(h2(w0 - ra.x, w1 - ra.y));
              pf[nt][gi][NQ - 1][1] = movmatrix(h2(w2 - rb.x, w3 - rb.y));
            }
          }
        }
        // value codes: dimensions 4 g .. 4 g + 3 of each block, tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        const uint8_t* vr = vc + (16 * mt + 2 * t) * ROW + g * 2 * NB;
        uint32_t v0[NB / 2], v1[NB / 2], v2[NB / 2], v3[NB / 2];
        lds_words<NB / 2>(vr, v0);
        lds_words<NB / 2>(vr + ROW, v1);
        lds_words<NB / 2>(vr + 8 * ROW, v2);
        lds_words<NB / 2>(vr + 9 * ROW, v3);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const uint32_t sel = (j & 1) ? 0x7632 : 0x5410;
          const uint32_t va = __byte_perm(v0[j >> 1], v1[j >> 1], sel), vb = __byte_perm(v2[j >> 1], v3[j >> 1], sel);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t ua = w ? va >> 8 : va, ub = w ? vb >> 8 : vb;
            const uint32_t a0 = centred_lo(ua), a1 = centred_hi(ua), a2 = centred_lo(ub), a3 = centred_hi(ub);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if constexpr (SPLIT) {  // the instruction cuts its sums off, always towards zero: added to `o` rounded
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < NQ; ++p) mma16816(sum, a0, a1, a2, a3, pf[nt][j / GB][p][0], pf[nt][j / GB][p][1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[nt][j][w][i] += sum[i];
              } else {
                mma16816(o[nt][j][w], a0, a1, a2, a3, pf[nt][j / GB][0][0], pf[nt][j / GB][0][1]);
              }
            }
          }
        }
      }

    }

    __syncwarp();  // every lane has read the stage
    if (issued < tiles) {
      issue();
      look_up();
      ++issued;
    }
    if (++st == STAGES) {
      st = 0;
      phase ^= 1u;
    }
  }
  if (!ok) {
    *abort_flag = 1;
    record_error(a.err, FGQ_ERR_TIMEOUT);
    for (int i = done; i < issued; ++i) mbar_wait_bounded(&bar[i % STAGES], (uint32_t)(i / STAGES) & 1u, 1u << 16);
  }

  // join: each warp's rows to shared memory with its reference, over the ring (every copy has landed)
  __syncthreads();
  {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) {
          l[nt][u] += __shfl_xor_sync(FULL_MASK, l[nt][u], s);
#pragma unroll
          for (int i = 0; i < NG; ++i) olo[nt][i][u] += __shfl_xor_sync(FULL_MASK, olo[nt][i][u], s);
        }
        const int row = 8 * nt + 2 * t + u;
        // r in log2 units; its rounding goes into the sums (past 2^24 there are no fractions left to keep)
        const float ref = fminf(fmaxf(-nref[nt][u] * mul[nt][u], -AT_TOP), AT_TOP), lost = fmaf(-nref[nt][u], mul[nt][u], -ref);
        const float back = ex2(fabsf(lost) <= 1.0f ? lost : 0.0f) * pow2f(-(int)off);
        float* dst = jo + (warp * NR + row) * D;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int w = 0; w < 2; ++w)
            *reinterpret_cast<float2*>(dst + 32 * j + 4 * g + 2 * w) =
                make_float2(fmaf(o[nt][j][w][u], 512.0f, olo[nt][j / GB][u]) * back,  // 2^9: the codes' scale
                            fmaf(o[nt][j][w][2 + u], 512.0f, olo[nt][j / GB][u]) * back);
        if (g == 0) {
          js[(warp * NR + row) * 2] = nref[nt][u] == -AT_M0 ? AT_M0 : ref;
          js[(warp * NR + row) * 2 + 1] = l[nt][u] * back;
        }
      }
  }
  __syncthreads();
  // the block's rows: from all warps into the first one's place
  float bm = AT_M0, bl = 0.0f;  // of row threadIdx.x
  for (int i = threadIdx.x; i < NR * D; i += 32 * AT_WARPS) {
    const int row = i / D, d = i % D, r = r0 + row;
    if (r >= a.rows) break;
    float mm = AT_M0, ll = 0.0f, v = 0.0f;
#pragma unroll
    for (int w = 0; w < AT_WARPS; ++w) mm = fmaxf(mm, js[(w * NR + row) * 2]);
#pragma unroll
    for (int w = 0; w < AT_WARPS; ++w) {
      const float f = ex2(js[(w * NR + row) * 2] - mm);
      ll = fmaf(f, js[(w * NR + row) * 2 + 1], ll);
      v = fmaf(f, jo[(w * NR + row) * D + d], v);
    }
    const int64_t orow = out_row(a, b, head, r);
    if (a.cluster) {
      jo[row * D + d] = v;
    } else if (a.chunks == 1) {
      store_out(a, orow * D + d, normalise(v, ll));
    } else {
      a.part[(orow * a.chunks + ch) * D + d] = v;
      if (d == 0) {
        a.stats[(orow * a.chunks + ch) * 2] = mm;
        a.stats[(orow * a.chunks + ch) * 2 + 1] = ll;
      }
    }
  }
  if (a.cluster) {
    if (threadIdx.x < NR) {
#pragma unroll
      for (int w = 0; w < AT_WARPS; ++w) bm = fmaxf(bm, js[(w * NR + threadIdx.x) * 2]);
#pragma unroll
      for (int w = 0; w < AT_WARPS; ++w)
        bl = fmaf(ex2(js[(w * NR + threadIdx.x) * 2] - bm), js[(w * NR + threadIdx.x) * 2 + 1], bl);
    }
    __syncthreads();
    if (threadIdx.x < NR) {
      js[2 * threadIdx.x] = bm;
      js[2 * threadIdx.x + 1] = bl;
    }
    cluster_sync();
    join_cluster<NB, NR>(a, b, head, r0, jo, js, ch);
    cluster_sync();  // no block leaves while another may read its sums
  }
}

struct AttnKernel {
  fgq_status (*launch)(const AttnArgs&, unsigned blocks, cudaStream_t);
  int rows, per_sm;  // query rows of a block; blocks an SM holds
  bool clusters;     // chunks may join as a cluster
  // us of the launch and a block's start and end, of those again in each further wave, and the tokens per us that a block
  // takes in between (all SMs full): fitted to the times at 32 sequences of 2000 tokens and 16 of 16384, 8 kv heads;
  // they choose a plan and change no result
  float start_us, wave_us, rate;
};

// The kernel for head_dim = 32 nb, group = 32 gb, fp32 inputs (split) or not, `rows` query rows at hand.
AttnKernel attention_kernel_2(int gb, bool split, int rows);
AttnKernel attention_kernel_4(int gb, bool split, int rows);
AttnKernel attention_kernel_8(int gb, bool split, int rows);
// The kernel for many query rows (kv_prompt.cu), bf16 and fp16.
AttnKernel prompt_kernel(int head_dim, int group, int rows);

}  // namespace dec
}  // namespace fgq
