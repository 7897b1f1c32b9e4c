// The product of up to 8 or 16 columns of tokens with 4-bit weights, tokens held in shared memory.
//
// A block keeps its tokens' columns for all of K (up to 8 NT x K x 2 bytes) and takes a run of items of 16 rows.  The run's tiles
// are one sequence, tile columns of an item after one another, and its warps share it in equal parts, wherever those cut an
// item: each warp streams its part through a ring of AHEAD tiles of its own in shared memory, with no barrier until the end.  (Loads to
// registers that far ahead did not stay in flight: their waits have no names of their own in a loop with branches.)  An item
// that a warp has whole goes from registers to its outputs; the parts of a cut one meet in shared memory once the warps are through,
// in their order.
// Bound by the weights' bytes and, a little later, by instructions (a tile is 4 words of 8 codes a lane and row: an AND and a packed multiply-add
// a pair, a matrix instruction 16 columns).  Logits of 8 tokens, 4096 -> 131072, groups of 128: 49 us, 84% of the copy rate, issue slots 74%
// busy (67 with the ring of w4_rows.cuh).  64 tokens of 6 of 64 experts, 4096 -> 1536, groups of 64: hidden values 83 us (5.3 TB/s, 67% of the DRAM
// peak, issue slots 70% busy), down, whose tokens have two columns each, 65 (3.5 TB/s, 44%; 62%; with one 48).  Up to 24 warps of 80
// registers: that many loads in flight, at 28 to 118 bytes of spills in the gated form.
#pragma once

#include "w4_rows.cuh"

namespace fgq {
namespace w4 {

enum { MODE_LINEAR = 0, MODE_GATED = 1, MODE_DOWN = 2 };

struct ResidentArgs {
  Matrix w, up;  // up: of a gated layer
  TokenRows x;
  int items;  // where the host knows how many there are (MODE_LINEAR: it does), or 0
  // MODE_LINEAR
  const float* bias;
  void* y;
  int P, M, ytype;
  // the experts: items (unit, rows)
  const Unit* units;
  const Choice* choices;
  const int* nunits;
  float* h;     // [choice][hpitch]: MODE_GATED out, MODE_DOWN in
  int64_t hpitch;
  unsigned* top;  // [choice]: the largest magnitude of its h, as fp32 bits (zeros before MODE_GATED)
  float* z;  // MODE_DOWN: out, [choice][M]
  int cols;   // columns of tokens held
  int one;    // MODE_GATED: there is one token
  int early;  // the kernel before is this library's: weights may be loaded while it runs
};

constexpr int RES_SMEM = 226 * 1024;  // a kilobyte is left for what is not dynamic
// Warps of a block at most: 80 registers a thread, or 96 where two row tiles meet 16 columns.
constexpr int resident_warps(int mt, int nt) { return mt * nt >= 4 ? 20 : 24; }

// Tokens through registers to shared memory, by a whole block.  A function of its own, or its registers would be the kernel's.
template <int PARTS>
__device__ __noinline__ void load_tokens(const TokenRows& x, int count, int ct, int stage, uint8_t* smem) {
  constexpr int BATCH = PARTS == 3 ? 2 : 4;  // loads in flight
  const int n = ct * 16 * count, threads = (int)blockDim.x;
  for (int i0 = threadIdx.x; i0 < n; i0 += BATCH * threads) {
    Eight<PARTS> e[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * threads, j = i >> 4, kt = j / count, tok = j - kt * count;
      if (i < n) e[b].load(x, tok, kt * TILE_COLS + 8 * (i & 15));
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = i0 + b * threads, j = i >> 4, kt = j / count, tok = j - kt * count;
      if (i < n) e[b].store(smem + kt * stage, tok, i & 15);
    }
  }
}

// MT: 2 tiles of MODE_GATED, gate's and up's, else 1.
template <typename T, int MT, int NT, int PER, int PARTS, int MODE, int AHEAD>
__global__ void __launch_bounds__(32 * resident_warps(MT, NT)) resident_kernel(const __grid_constant__ ResidentArgs a) {
  constexpr int CPT = columns_per_token(PARTS), TOKENS = 8 * NT / CPT, COLS = 8 * NT;
  const int STAGE = a.cols * 256;  // bytes of a tile column's tokens
  static_assert(MT == (MODE == MODE_GATED ? 2 : 1), "tiles of an item");
  constexpr int LD = 16 * MT + 1, FRAGMENT = COLS * LD, TB = tile_bytes<PER>(), SLOT = MT * TB;
  extern __shared__ __align__(16) uint8_t w4_smem[];
  __shared__ int row_of[TOKENS];    // MODE_GATED: the tokens' rows
  __shared__ float back[TOKENS];    // MODE_DOWN: what the tokens' scales are undone by
  __shared__ unsigned tops[TOKENS];  // MODE_GATED: the tokens' largest hidden values in this block
  const int W = (int)blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int ct = a.w.ct;
  uint8_t* ring = w4_smem + ct * STAGE + warp * AHEAD * SLOT;
  const uint32_t ring_at = smem_u32(ring);
  float* sums = reinterpret_cast<float*>(w4_smem + ct * STAGE + W * AHEAD * SLOT);  // [warp][first, last][column][LD]
  if (MODE == MODE_GATED) {
    pdl_wait();
    pdl_trigger();  // from here on the kernel after may read the units
  } else if (MODE == MODE_DOWN) {
    pdl_trigger();
  }
  const int rt = a.w.rt;  // items of a unit
  const int items = MODE == MODE_LINEAR || a.items > 0 ? a.items : __ldcg(a.nunits) * rt;
  int i0, i1;
  const int units = items / rt;
  // a few units: equal blocks each, as a run that crosses into the next unit has its tokens to wait for (one token, 8 experts of 64 2048 -> 1024
  // 21.8 us without and 20.5; two tokens 29.5 and 25.6)
  if (MODE != MODE_LINEAR && units > 0 && 2 * units <= (int)gridDim.x) {
    const int blocks = (int)gridDim.x / units, run = (rt + blocks - 1) / blocks, unit = (int)blockIdx.x / blocks, j = (int)blockIdx.x - unit * blocks;
    i0 = unit * rt + min(j * run, rt);
    i1 = unit < units ? unit * rt + min((j + 1) * run, rt) : 0;
  } else {
    const int run = (items + (int)gridDim.x - 1) / (int)gridDim.x;
    i0 = (int)blockIdx.x * run;
    i1 = min(i0 + run, items);
  }
  if (i0 >= i1) {
    // a block without items may be any, or all where no choice is an expert: what comes after this kernel comes after the one before
    if (MODE == MODE_DOWN || (MODE == MODE_LINEAR && a.early)) pdl_wait();
    return;
  }

  // a segment: the run's items of one unit
  struct Segment {
    int item, count;   // first item (of the unit's), items
    int4 u;            // expert, first choice, how many
    int each, more;    // tiles of a warp, of the first `more` one more
    int q0, q1;        // this warp's tiles of the segment's count * ct
    __device__ __forceinline__ int begins(int w) const { return w * each + min(w, more); }
  };
  auto segment_at = [&](int i) {
    Segment s;
    if (MODE == MODE_LINEAR) {
      s.item = i;
      s.count = i1 - i;
      s.u = make_int4(0, 0, min(TOKENS, a.P), 0);
    } else {
      const int unit = i / rt;
      s.item = i - unit * rt;
      s.count = min(i1 - i, rt - s.item);
      s.u = __ldcg(reinterpret_cast<const int4*>(a.units) + unit);
    }
    s.each = s.count * ct / W;
    s.more = s.count * ct - s.each * W;
    s.q0 = s.begins(warp);
    s.q1 = s.begins(warp + 1);
    return s;
  };
  // the next tile to load: its codes and scales, 16 bytes on a lane, and where it goes
  const uint8_t *codes = nullptr, *scales = nullptr;
  const int64_t up_codes = MODE == MODE_GATED ? a.up.codes - a.w.codes : 0;
  const int64_t up_scales = MODE == MODE_GATED ? reinterpret_cast<const uint8_t*>(a.up.scales) - reinterpret_cast<const uint8_t*>(a.w.scales) : 0;
  int left = 0;
  const uint32_t ring0 = ring_at + 16 * lane;
  auto begin = [&](const Segment& s) {
    const int64_t at = ((int64_t)s.u.x * rt + s.item) * ct + s.q0;  // an item's tiles follow the last's
    codes = a.w.codes + at * TILE_BYTES + 16 * lane;
    scales = reinterpret_cast<const uint8_t*>(a.w.scales) + at * (TILE_ROWS * PER * 2) + 16 * lane;
    left = s.q1 - s.q0;
  };
  auto load = [&](int slot) {
    const uint32_t to = ring0 + slot * SLOT;
    if (left > 0) {
      --left;
      copy_tile<PER>(to, codes, scales, lane);
      if (MODE == MODE_GATED) copy_tile<PER>(to + TB, codes + up_codes, scales + up_scales, lane);
      codes += TILE_BYTES;
      scales += TILE_ROWS * PER * 2;
    }
    cp_async_commit();
  };
  Segment now = segment_at(i0);
  begin(now);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(i);
  if (MODE == MODE_DOWN || (MODE == MODE_LINEAR && a.early)) pdl_wait();

  const uint8_t* xb = static_cast<const uint8_t*>(a.x.data);
  const uint32_t xs = smem_u32(w4_smem);
  // the segment's columns, 16 bytes a thread and turn; columns of no token are left as they are: nothing reads their sums
  auto tokens = [&]() {
    if constexpr (MODE == MODE_DOWN) {
      // fp32 values in fp16 parts (fp32 outputs: bf16 ones, which need no scale), after a power of two that takes the token's largest
      // to 2^14: two parts are within 2^-22 of a value, or 2^-39 of the largest; three exact.  (One part, within 2^-12, left bf16
      // outputs 9e-4 of their norm from those of exact values rounded once, across whose borders it takes them; their own rounding is 1.7e-3.)
      const int pieces = ct * 16, n = pieces * now.u.z;
      for (int i = threadIdx.x; i < n; i += 32 * W) {
        const int tok = i / pieces, j = i - tok * pieces, k = 8 * j;
        float v[8], up = 1.0f, up2 = 1.0f;
        if (PARTS < 3) {
          const unsigned big = __ldcg(a.top + now.u.y + tok);
          const int e = max((int)(big >> 23) - 127, -126);
          up = pow2f((14 - e) / 2), up2 = pow2f((14 - e) - (14 - e) / 2);  // past fp32's largest for tiny ones
          if (j == 0) back[tok] = e == 128 ? 1.0f : pow2f(e - 14);
          if (e == 128) up = up2 = 1.0f;  // NaN or infinity
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (k < a.hpitch) f = __ldcg(reinterpret_cast<const float4*>(a.h + (now.u.y + tok) * a.hpitch + k) + h);
          v[4 * h] = f.x, v[4 * h + 1] = f.y, v[4 * h + 2] = f.z, v[4 * h + 3] = f.w;
        }
        uint32_t w[3][4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          if constexpr (PARTS == 3) {
            uint16_t p[3], q[3];
            three_parts(v[2 * h], p);
            three_parts(v[2 * h + 1], q);
#pragma unroll
            for (int c = 0; c < 3; ++c) w[c][h] = p[c] | (uint32_t)q[c] << 16;
          } else {
            const float x0 = v[2 * h] * up * up2, x1 = v[2 * h + 1] * up * up2;
            w[0][h] = pack2(x0, x1, __half());
            if constexpr (PARTS == 2) {
              const float2 r = unpack2(w[0][h], __half());
              w[1][h] = pack2(x0 - r.x, x1 - r.y, __half());
            }
          }
        }
#pragma unroll
        for (int c = 0; c < CPT; ++c)
          *reinterpret_cast<uint4*>(w4_smem + (j >> 4) * STAGE + chunk_at(tok * CPT + c, j & 15)) =
              c < PARTS ? make_uint4(w[c < PARTS ? c : 0][0], w[c < PARTS ? c : 0][1], w[c < PARTS ? c : 0][2], w[c < PARTS ? c : 0][3])
                        : make_uint4(0u, 0u, 0u, 0u);
      }
      __syncthreads();
      return;
    }
    if (MODE == MODE_GATED && !a.one) {
      if (threadIdx.x < now.u.z) row_of[threadIdx.x] = __ldcg(&a.choices[now.u.y + threadIdx.x].token);
      __syncthreads();
    }
    // pieces of 16 bytes as they are; the experts' fp32 tokens: three rows of bf16 parts beside one another
    if (MODE == MODE_GATED || (PARTS == 1 && a.x.load == ROWS_COPIED)) {
      const int cols = now.u.z * CPT, n = ct * 16 * cols;
      for (int i = threadIdx.x; i < n; i += 32 * W) {
        const int chunk = i & 15, j = i >> 4, kt = j / cols, c = j - kt * cols, tok = c / CPT, part = c % CPT, k = kt * TILE_COLS + 8 * chunk;
        const int64_t row = MODE == MODE_LINEAR ? tok : (a.one ? 0 : row_of[tok]);
        const bool live = part < PARTS && k < a.x.kvalid;
        cp_async16(xs + kt * STAGE + chunk_at(c, chunk), live ? xb + 2 * (row * a.x.pitch + part * (a.x.pitch / PARTS) + k) : xb, live ? 16u : 0u);
      }
      cp_async_commit();
      cp_async_wait<0>();
    } else if constexpr (MODE == MODE_LINEAR) {
      load_tokens<PARTS>(a.x, now.u.z, ct, STAGE, w4_smem);
    }
    __syncthreads();
  };
  // what becomes of the finished sums of row r of an item and token tok: of gate and up, or of one matrix.  MODE_GATED: the
  // hidden value's magnitude
  auto finish = [&](int item, int r, int tok, float v, float u) {
    const int m = item * TILE_ROWS + r;
    v *= Operand<T>::BACK;
    if (MODE == MODE_GATED) {
      u *= Operand<T>::BACK;
      const float f = m < a.M ? v / (1.0f + expf(-v)) * u : 0.0f;
      a.h[(now.u.y + tok) * a.hpitch + m] = f;
      return fabsf(f);
    }
    if (m < a.M) {
      if (MODE == MODE_DOWN)
        a.z[(int64_t)(now.u.y + tok) * a.M + m] = PARTS < 3 ? v * back[tok] : v;
      else
        store_typed(a.y, a.ytype, (int64_t)tok * a.M + m, v + (a.bias ? __ldg(a.bias + m) : 0.0f));
    }
    return 0.0f;
  };
  // a token's largest hidden value: of this lane's two tokens in registers, a segment long, then of the block, then of all (an
  // atomic a warp and item took the hidden layer of 16 tokens from 48 to 86 us).  Magnitudes compare as whole numbers, NaN
  // above all, and the order does not matter
  constexpr bool TOPS = MODE == MODE_GATED && CPT == 1;
  unsigned big[NT][2];
  auto note = [&](int tok, float f) { atomicMax(tops + tok, __float_as_uint(f)); };

  const Pieces<NT> pieces(a.cols, lane);
  pair_t sum[MT][NT][2];
  auto clear = [&]() {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sum[mt][nt][0] = sum[mt][nt][1] = 0ull;
  };
  // this lane's sums as those of tokens
  auto whole = [&](int item) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float s[2], u[2];
        unpack_f2(sum[0][nt][half], s[0], s[1]);
        unpack_f2(sum[MT - 1][nt][half], u[0], u[1]);
        const int r = g + 8 * half;
        if constexpr (CPT == 1) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (8 * nt + 2 * t + e < now.u.z) big[nt][e] = max(big[nt][e], __float_as_uint(finish(item, r, 8 * nt + 2 * t + e, s[e], u[e])));
        } else if constexpr (CPT == 2) {
          if (4 * nt + t < now.u.z) finish(item, r, 4 * nt + t, s[0] + s[1], u[0] + u[1]);
        } else {  // three parts, and a column that is zero
          float v = s[0] + s[1], w = u[0] + u[1];
          v += __shfl_xor_sync(FULL_MASK, v, 1);
          if (MODE == MODE_GATED) w += __shfl_xor_sync(FULL_MASK, w, 1);
          const int tok = 2 * nt + (t >> 1);
          if ((t & 1) == 0 && tok < now.u.z) finish(item, r, tok, v, w);
        }
      }
    }
  };
  auto fragment = [&](int slot) {
    float* to = sums + (2 * warp + slot) * FRAGMENT;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float s0, s1;
          unpack_f2(sum[mt][nt][half], s0, s1);
          to[(8 * nt + 2 * t) * LD + 16 * mt + g + 8 * half] = s0;
          to[(8 * nt + 2 * t + 1) * LD + 16 * mt + g + 8 * half] = s1;
        }
  };

  for (int i = i0;;) {
    if (TOPS) {
      if (threadIdx.x < TOKENS) tops[threadIdx.x] = 0u;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) big[nt][0] = big[nt][1] = 0u;
    }
    tokens();
    clear();
    int item = now.q0 / ct, kt = now.q0 - item * ct;
    const int first = item;
    bool cut = kt > 0;  // whether the item began in the warp before
    const uint8_t* stage = w4_smem + kt * STAGE;
    for (int q = now.q1 - now.q0; q > 0;) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {  // a segment begins with the ring's first tile
        if (q == 0) break;
        --q;
        cp_async_wait<AHEAD - 1>();
        __syncwarp();  // every lane's part of the tile is there
        Tile<PER> tile[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) read_tile<PER>(tile[mt], ring + k * SLOT + mt * TB, lane);
        multiply<T, MT, NT, PER>(tile, stage, pieces, sum);
        __syncwarp();  // and read
        load(k);
        stage += STAGE;
        if (++kt == ct) {
          if (cut)
            fragment(0);
          else
            whole(now.item + item);
          clear();
          cut = false;
          kt = 0;
          stage = w4_smem;
          ++item;
        }
      }
    }
    if (kt > 0 && now.q1 > now.q0) fragment(item == first ? 0 : 1);
    if constexpr (TOPS) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tok = 8 * nt + 2 * t + e;
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) big[nt][e] = max(big[nt][e], __shfl_xor_sync(FULL_MASK, big[nt][e], o));
          if (g == 0 && tok < now.u.z) note(tok, __uint_as_float(big[nt][e]));
        }
    }
    // the next segment's first tiles
    i += now.count;
    Segment next = now;
    if (i < i1) {
      next = segment_at(i);
      begin(next);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) load(k);
    }
    __syncthreads();
    // a cut item is put together by the first warp whose part begins inside it
    constexpr int ROWS = TILE_ROWS;
    const int it = now.q0 / ct, lo = it * ct, hi = lo + ct;
    if (warp > 0 && now.q0 > lo && now.q0 < now.q1 && now.begins(warp - 1) <= lo) {
      int last = warp;  // the last warp with a part of it
      while (last + 1 < W && now.begins(last + 1) < hi && now.begins(last + 1) < now.begins(last + 2)) ++last;
      for (int j = lane; j < now.u.z * ROWS; j += 32) {
        const int tok = j / ROWS, r = j % ROWS;
        float v = 0.0f, u = 0.0f;
        for (int k = warp - 1; k <= last; ++k) {
          const float* from = sums + (2 * k + (now.begins(k) >= lo ? 0 : 1)) * FRAGMENT + tok * CPT * LD + r;
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            v += from[part * LD];
            if (MODE == MODE_GATED) u += from[part * LD + 16];
          }
        }
        const float f = finish(now.item + it, r, tok, v, u);
        if (TOPS) note(tok, f);
      }
    }
    if (TOPS) {
      __syncthreads();
      if ((int)threadIdx.x < now.u.z) atomicMax(a.top + now.u.y + threadIdx.x, tops[threadIdx.x]);
    }
    if (i >= i1) break;
    __syncthreads();  // the parts are read, and the tokens
    now = next;
  }
}

// How a block holds its tokens: one block an SM, its warps, its shared memory.
struct ResidentPlan {
  int warps, smem, cols;
};
// warps = 0: the tokens do not fit beside eight warps' rings.
template <int MT, int NT, int AHEAD>
ResidentPlan plan_resident(int ct, int per, int cols) {
  const int64_t x = (int64_t)ct * cols * 256;
  const int tile = TILE_BYTES + TILE_ROWS * per * 2;
  const int each = AHEAD * MT * tile + 2 * 8 * NT * (16 * MT + 1) * 4;
  const int64_t room = (RES_SMEM - x) / each;
  const int warps = room > resident_warps(MT, NT) ? resident_warps(MT, NT) : (int)room;
  if (warps < 8) return {0, 0, 0};
  return {warps, (int)(x + (int64_t)warps * each), cols};
}

template <typename T, int MT, int NT, int PER, int PARTS, int MODE, int AHEAD>
fgq_status launch_resident(ResidentArgs a, const ResidentPlan& plan, int64_t items, bool chained, cudaStream_t s) {
  a.cols = plan.cols;
  constexpr auto kernel = resident_kernel<T, MT, NT, PER, PARTS, MODE, AHEAD>;
  if (!tc::smem_attr_once<resident_kernel<T, MT, NT, PER, PARTS, MODE, AHEAD>>(RES_SMEM)) return FGQ_ERR_CUDA;
  const int64_t most = device_sms(), run = (items + most - 1) / most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(MODE == MODE_LINEAR ? (items + run - 1) / run : (items < most ? items : most)));
  cfg.blockDim = dim3(32 * plan.warps);
  cfg.dynamicSmemBytes = plan.smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = chained ? 1 : 0;
  return after_launch(cudaLaunchKernelEx(&cfg, kernel, a));
}

}  // namespace w4
}  // namespace fgq
