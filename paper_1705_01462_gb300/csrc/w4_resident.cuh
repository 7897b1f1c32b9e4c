// The product of up to 8 or 16 columns of tokens with 4-bit weights, tokens held in shared memory.
//
// A block keeps its tokens' columns for all of K (8 NT x K x 2 bytes) and takes a run of items of 16 MT rows.  The run's tiles
// are one sequence, tile columns of an item after one another, and its warps share it in equal parts, wherever those cut an
// item: each warp streams its part through a ring of AHEAD tiles of its own in shared memory, with no barrier until the end.  (Loads to
// registers that far ahead did not stay in flight: their waits have no names of their own in a loop with branches.)  An item
// that a warp has whole goes from registers to its outputs; the parts of a cut one meet in shared memory once the warps are through,
// in their order.
#pragma once

#include "w4_rows.cuh"

namespace fgq {
namespace w4 {

enum { MODE_LINEAR = 0, MODE_GATED = 1, MODE_DOWN = 2 };

struct ResidentArgs {
  Matrix w, up;  // up: of a gated layer
  TokenRows x;
  // MODE_LINEAR
  const float* bias;
  void* y;
  int P, M, ytype, items;
  // the experts: items (unit, rows)
  const Unit* units;
  const Choice* choices;
  const int* nunits;
  uint16_t* h;  // MODE_GATED: out, [choice][parts][hpitch]
  int64_t hpitch;
  float* z;  // MODE_DOWN: out, [choice][M]
  int one;    // MODE_GATED: there is one token
  int early;  // the kernel before is this library's: weights may be loaded while it runs
};

constexpr int RES_MAX_WARPS = 24, RES_SMEM = 226 * 1024;  // a kilobyte is left for what is not dynamic

template <typename T, int MT, int NT, int PER, int PARTS, int MODE, int HPARTS, int AHEAD>
__global__ void __launch_bounds__(32 * RES_MAX_WARPS) resident_kernel(const __grid_constant__ ResidentArgs a) {
  constexpr int CPT = columns_per_token(PARTS), TOKENS = 8 * NT / CPT, COLS = 8 * NT, STAGE = COLS * 256;
  constexpr int TILES = MODE == MODE_GATED ? 1 : MT;  // row tiles of an item
  constexpr int LD = 16 * MT + 1, FRAGMENT = COLS * LD, TB = tile_bytes<PER>(), SLOT = MT * TB;
  extern __shared__ __align__(16) uint8_t w4_smem[];
  __shared__ int row_of[TOKENS];
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
  const int groups = (a.w.rt + TILES - 1) / TILES;  // items of a unit
  const int items = MODE == MODE_LINEAR ? a.items : __ldcg(a.nunits) * groups;
  const int run = (items + (int)gridDim.x - 1) / (int)gridDim.x;
  const int i0 = (int)blockIdx.x * run, i1 = min(i0 + run, items);
  if (i0 >= i1) return;

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
      const int unit = i / groups;
      s.item = i - unit * groups;
      s.count = min(i1 - i, groups - s.item);
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
  int lkt = 0, lrow = 0, left = 0;
  const uint32_t ring0 = ring_at + 16 * lane, ring_end = ring0 + AHEAD * SLOT;
  uint32_t to = ring0;
  auto begin = [&](const Segment& s) {
    const int i = s.q0 / ct;
    lkt = s.q0 - i * ct;
    lrow = (s.item + i) * TILES;
    const int64_t at = ((int64_t)s.u.x * a.w.rt + lrow) * ct + lkt;
    codes = a.w.codes + at * TILE_BYTES + 16 * lane;
    scales = reinterpret_cast<const uint8_t*>(a.w.scales) + at * (TILE_ROWS * PER * 2) + 16 * lane;
    left = s.q1 - s.q0;
  };
  auto load = [&]() {
    if (left > 0) {
      --left;
      copy_tile<PER>(to, codes, scales, lane);
      if (MODE == MODE_GATED) {
        copy_tile<PER>(to + TB, codes + up_codes, scales + up_scales, lane);
      } else {
#pragma unroll
        for (int mt = 1; mt < MT; ++mt) {  // a row tile past the last is read as the last
          const int64_t on = lrow + mt < a.w.rt ? (int64_t)mt * ct : 0;
          copy_tile<PER>(to + mt * TB, codes + on * TILE_BYTES, scales + on * (TILE_ROWS * PER * 2), lane);
        }
      }
      to = to + SLOT == ring_end ? ring0 : to + SLOT;
      codes += TILE_BYTES;
      scales += TILE_ROWS * PER * 2;
      if (TILES > 1 && ++lkt == ct) {
        lkt = 0;
        lrow += TILES;
        codes += (int64_t)(TILES - 1) * ct * TILE_BYTES;
        scales += (int64_t)(TILES - 1) * ct * (TILE_ROWS * PER * 2);
      }
    }
    cp_async_commit();
  };
  Segment now = segment_at(i0);
  begin(now);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load();
  if (MODE == MODE_DOWN || (MODE == MODE_LINEAR && a.early)) pdl_wait();

  const uint8_t* xb = static_cast<const uint8_t*>(a.x.data);
  const uint32_t xs = smem_u32(w4_smem);
  // the segment's columns, 16 bytes a thread and turn; columns of no token are left as they are: nothing reads their sums
  auto tokens = [&]() {
    if (MODE == MODE_GATED && !a.one) {
      if (threadIdx.x < now.u.z) row_of[threadIdx.x] = __ldcg(&a.choices[now.u.y + threadIdx.x].token);
      __syncthreads();
    }
    const int cols = now.u.z * CPT, n = ct * 16 * cols;
    for (int i = threadIdx.x; i < n; i += 32 * W) {
      const int chunk = i & 15, j = i >> 4, kt = j / cols, c = j - kt * cols, tok = c / CPT, part = c % CPT, k = kt * TILE_COLS + 8 * chunk;
      const int64_t row = MODE == MODE_LINEAR ? tok : (MODE == MODE_GATED ? (a.one ? 0 : row_of[tok]) : now.u.y + tok);
      const bool live = part < PARTS && k < a.x.kvalid;
      cp_async16(xs + kt * STAGE + chunk_at(c, chunk), live ? xb + 2 * (row * a.x.pitch + part * (a.x.pitch / PARTS) + k) : xb, live ? 16u : 0u);
    }
    cp_async_commit();
    cp_async_wait<0>();
    __syncthreads();
  };
  // what becomes of the finished sums of row r of an item and token tok: of gate and up, or of one matrix
  auto finish = [&](int item, int r, int tok, float v, float u) {
    const int m = item * 16 * TILES + r;
    v *= Operand<T>::BACK;
    if (MODE == MODE_GATED) {
      u *= Operand<T>::BACK;
      const float f = m < a.M ? v / (1.0f + expf(-v)) * u : 0.0f;
      uint16_t p[3];
      hidden_parts<HPARTS>(f, p);
      uint16_t* to = a.h + (int64_t)(now.u.y + tok) * HPARTS * a.hpitch + m;
#pragma unroll
      for (int part = 0; part < HPARTS; ++part) to[part * a.hpitch] = p[part];
    } else if (m < a.M) {
      if (MODE == MODE_DOWN)
        a.z[(int64_t)(now.u.y + tok) * a.M + m] = v;
      else
        store_typed(a.y, a.ytype, (int64_t)tok * a.M + m, v + (a.bias ? __ldg(a.bias + m) : 0.0f));
    }
  };

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
    for (int mt = 0; mt < TILES; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float s[2], u[2];
          unpack_f2(sum[mt][nt][half], s[0], s[1]);
          unpack_f2(sum[MODE == MODE_GATED ? MT - 1 : mt][nt][half], u[0], u[1]);
          const int r = 16 * mt + g + 8 * half;
          if constexpr (CPT == 1) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (8 * nt + 2 * t + e < now.u.z) finish(item, r, 8 * nt + 2 * t + e, s[e], u[e]);
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

  const uint8_t* from = ring;  // of the next tile to multiply
  for (int i = i0;;) {
    tokens();
    clear();
    int item = now.q0 / ct, kt = now.q0 - item * ct;
    const int first = item;
    bool cut = kt > 0;  // whether the item began in the warp before
    const uint8_t* stage = w4_smem + kt * STAGE;
#pragma unroll 1
    for (int q = now.q1 - now.q0; q > 0; --q) {
      cp_async_wait<AHEAD - 1>();
      __syncwarp();  // every lane's part of the tile is there
      Tile<PER> tile[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) read_tile<PER>(tile[mt], from + mt * TB, lane);
      multiply<T, MT, NT, PER>(tile, stage, sum, lane);
      __syncwarp();  // and read
      load();
      from = from + SLOT == ring + AHEAD * SLOT ? ring : from + SLOT;
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
    if (kt > 0 && now.q1 > now.q0) fragment(item == first ? 0 : 1);
    // the next segment's first tiles
    i += now.count;
    Segment next = now;
    if (i < i1) {
      next = segment_at(i);
      begin(next);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) load();
    }
    __syncthreads();
    // a cut item is put together by the first warp whose part begins inside it
    constexpr int ROWS = 16 * TILES;
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
        finish(now.item + it, r, tok, v, u);
      }
    }
    if (i >= i1) break;
    __syncthreads();  // the parts are read, and the tokens
    now = next;
  }
}

// How a block holds its tokens: one block an SM, its warps, its shared memory.
struct ResidentPlan {
  int warps, smem;
};
// warps = 0: the tokens do not fit beside eight warps' rings.
template <int MT, int NT, int AHEAD>
ResidentPlan plan_resident(int ct, int per) {
  const int64_t x = (int64_t)ct * 8 * NT * 256;
  const int tile = TILE_BYTES + TILE_ROWS * per * 2;
  const int each = AHEAD * MT * tile + 2 * 8 * NT * (16 * MT + 1) * 4;
  const int64_t room = (RES_SMEM - x) / each;
  const int warps = room > RES_MAX_WARPS ? RES_MAX_WARPS : (int)room;
  if (warps < 8) return {0, 0};
  return {warps, (int)(x + (int64_t)warps * each)};
}

template <typename T, int MT, int NT, int PER, int PARTS, int MODE, int HPARTS, int AHEAD>
fgq_status launch_resident(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, bool chained, cudaStream_t s) {
  constexpr auto kernel = resident_kernel<T, MT, NT, PER, PARTS, MODE, HPARTS, AHEAD>;
  if (!tc::smem_attr_once<resident_kernel<T, MT, NT, PER, PARTS, MODE, HPARTS, AHEAD>>(RES_SMEM)) return FGQ_ERR_CUDA;
  const int64_t most = device_sms(), run = (items + most - 1) / most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((items + run - 1) / run));
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
