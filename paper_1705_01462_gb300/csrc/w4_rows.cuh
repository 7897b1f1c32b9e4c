// The product of few tokens with 4-bit weights, and with two matrices at once for a gated layer.
#pragma once

#include "linear_internal.cuh"
#include "w4.cuh"

namespace fgq {
namespace w4 {

// A unit of work of the experts: up to `cap` choices of one expert, `count` of them from `start` on in the order sorted by expert.
struct Unit {
  int expert, start, count, pad;
};
// A choice in that order: its token and the router's weight.
struct Choice {
  int token;
  float weight;
};

// v as PARTS bf16 values that add up to it: all of it in three, within 2^-17 in two.
template <int PARTS>
__device__ __forceinline__ void hidden_parts(float v, uint16_t (&p)[3]) {
  if constexpr (PARTS == 3) {
    three_parts(v, p);
  } else {
    const float a = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    const __nv_bfloat16 b = __float2bfloat16_rn(v - a);
    p[0] = (uint16_t)(__float_as_uint(a) >> 16);
    p[1] = *reinterpret_cast<const uint16_t*>(&b);
  }
}

struct RowsArgs {
  Matrix w, up;  // up: of a gated layer
  TokenRows x;
  int splits;  // blocks of a cluster that share K
  // a linear layer: items (rows, tokens), the tokens' tiles first
  const float* bias;
  void* y;
  int P, M, ytype, items, token_tiles;
  // a gated layer: items (unit, rows)
  const Unit* units;
  const Choice* choices;
  const int* nunits;
  uint16_t* h;  // [choice][parts][hpitch], in sorted order
  int64_t hpitch;
  int early;  // the kernel before is this library's: weights may be loaded while it runs
};

// GATED: tile 0 of gate and tile 1 of up, hidden values left in HPARTS parts.  Otherwise MT tiles of w, and y.
template <typename T, int MT, int NT, int PER, int PARTS, bool GATED, int HPARTS, int AHEAD>
__global__ void __launch_bounds__(THREADS) rows_kernel(const __grid_constant__ RowsArgs a) {
  using R = Ring<NT>;
  constexpr int CPT = columns_per_token(PARTS), TOKENS = 8 * NT / CPT;
  constexpr int GROUP = GATED ? WARPS : WARPS * MT;  // row tiles of an item
  extern __shared__ __align__(16) uint8_t w4_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (GATED) {
    pdl_wait();
    pdl_trigger();  // from here on the kernel after may read the units
  }
  const int groups = (a.w.rt + GROUP - 1) / GROUP;
  int items, sp = 0, i0, i1;
  if (GATED)
    items = __ldcg(a.nunits) * groups;
  else
    items = a.items;
  if (a.splits > 1) {  // one item a cluster
    sp = blockIdx.x % a.splits;
    i0 = blockIdx.x / a.splits;
    i1 = i0 + 1;
  } else {  // equal runs of items
    const int run = (items + (int)gridDim.x - 1) / (int)gridDim.x;
    i0 = (int)blockIdx.x * run;
    i1 = min(i0 + run, items);
  }
  if (i0 >= items) return;  // a whole cluster
  const int c0 = (int)((int64_t)a.w.ct * sp / a.splits), c1 = (int)((int64_t)a.w.ct * (sp + 1) / a.splits), ct = c1 - c0;
  const int64_t n = (int64_t)(i1 - i0) * ct;  // stages

  // what an item is
  struct Item {
    int64_t first;       // its first tile's number for this warp (GATED: of either matrix)
    int rt, tok0, count;  // row tile of this warp, first token (choice), how many there are
  };
  auto item_at = [&](int i) {
    Item it;
    if (GATED) {
      const int u = i / groups, rg = i - u * groups;
      const int4 v = __ldcg(reinterpret_cast<const int4*>(a.units) + u);
      it.rt = rg * GROUP + warp;
      it.first = ((int64_t)v.x * a.w.rt + min(it.rt, a.w.rt - 1)) * a.w.ct + c0;
      it.tok0 = v.y;
      it.count = v.z;
    } else {
      const int rg = i / a.token_tiles, tt = i - rg * a.token_tiles;
      it.rt = rg * GROUP + warp * MT;
      it.first = (int64_t)it.rt * a.w.ct + c0;
      it.tok0 = tt * TOKENS;
      it.count = min(TOKENS, a.P - it.tok0);
    }
    return it;
  };
  Tile<PER> tile[AHEAD][MT];
  auto weights = [&](int slot, const Item& it, int kt) {
    if (GATED) {
      tile[slot][0].load(a.w.codes, a.w.scales, it.first + kt, lane);
      tile[slot][1].load(a.up.codes, a.up.scales, it.first + kt, lane);
    } else {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {  // a row tile past the last is read as the last
        const int64_t back = (int64_t)max(it.rt + mt - (a.w.rt - 1), 0) - mt;
        tile[slot][mt].load(a.w.codes, a.w.scales, it.first - back * a.w.ct + kt, lane);
      }
    }
  };
  Columns<NT> cols;
  auto columns = [&](const Item& it) {
#pragma unroll
    for (int i = 0; i < R::COPIES; ++i) {
      const int col = (int)(threadIdx.x >> 4) + 16 * i, tok = col / CPT, part = col % CPT;
      cols.off[i] = -1;
      if (tok < it.count && part < PARTS) {
        const int row = GATED ? __ldcg(&a.choices[it.tok0 + tok].token) : it.tok0 + tok;
        cols.off[i] = 2 * (row * a.x.pitch + part * (a.x.pitch / PARTS));
      }
    }
  };

  const uint8_t* xb = static_cast<const uint8_t*>(a.x.data);
  const uint32_t ring_at = smem_u32(w4_smem);
  // three places in the sequence of stages: the weights to load, the tokens to copy, and the stage to multiply
  Item now = item_at(i0), wit = now, xit = now;
  int kt = 0, wi = i0, wkt = 0, xi = i0, xkt = 0, xslot = 0, slot = 0;
  auto next_weights = [&](int at) {
    weights(at, wit, wkt);
    if (++wkt == ct) {
      wkt = 0;
      if (++wi < i1) wit = item_at(wi);
    }
  };
  auto next_tokens = [&]() {
    cols.copy(ring_at + xslot * R::BYTES, xb, c0 + xkt, a.x.kvalid);
    xslot = xslot + 1 == R::STAGES ? 0 : xslot + 1;
    if (++xkt == ct) {
      xkt = 0;
      if (++xi < i1) {
        xit = item_at(xi);
        columns(xit);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < n) next_weights(i);
  if (!GATED && a.early) pdl_wait();
  columns(xit);
#pragma unroll
  for (int i = 0; i < R::STAGES - 1; ++i) {
    if (i < n) next_tokens();
    cp_async_commit();
  }
  pair_t sum[MT][NT][2];
  auto clear = [&]() {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sum[mt][nt][0] = sum[mt][nt][1] = 0ull;
  };
  clear();

  // what becomes of a finished sum of row r (of the item's row tile) and token tok: gate's and up's, or one of the MT tiles'
  auto finish = [&](const Item& it, int rt, int r, int tok, float v, float w) {
    const int m = rt * TILE_ROWS + r;
    if (GATED) {
      v *= Operand<T>::BACK;
      w *= Operand<T>::BACK;
      if (rt >= a.w.rt) return;
      const float z = m < a.M ? v / (1.0f + expf(-v)) * w : 0.0f;
      uint16_t p[3];
      hidden_parts<HPARTS>(z, p);
      uint16_t* to = a.h + (int64_t)(it.tok0 + tok) * HPARTS * a.hpitch + m;
#pragma unroll
      for (int part = 0; part < HPARTS; ++part) to[part * a.hpitch] = p[part];
    } else {
      if (m < a.M)
        store_typed(a.y, a.ytype, (int64_t)(it.tok0 + tok) * a.M + m, fmaf(v, Operand<T>::BACK, a.bias ? __ldg(a.bias + m) : 0.0f));
    }
  };
  // this lane's sums of one tile and eight columns as those of tokens: value (row g or g + 8) of token `tok`, or none
  auto each = [&](const Item& it, int mt, auto f) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float s[2], u[2];
        unpack_f2(sum[mt][nt][half], s[0], s[1]);
        unpack_f2(sum[GATED ? MT - 1 : mt][nt][half], u[0], u[1]);
        if constexpr (CPT == 1) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (8 * nt + 2 * t + e < it.count) f(g + 8 * half, 8 * nt + 2 * t + e, s[e], u[e]);
        } else {  // three parts, and a column that is zero
          float v = s[0] + s[1], w = u[0] + u[1];
          v += __shfl_xor_sync(FULL_MASK, v, 1);
          if (GATED) w += __shfl_xor_sync(FULL_MASK, w, 1);
          const int tok = 2 * nt + (t >> 1);
          if ((t & 1) == 0 && tok < it.count) f(g + 8 * half, tok, v, w);
        }
      }
  };

  const Pieces<NT> pieces(8 * NT, lane);
  for (int64_t q = 0; q < n; q += AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (q + i >= n) break;  // the same for the whole block
      cp_async_wait<R::STAGES - 2>();
      __syncthreads();  // the stage is there for everyone, and the one before has been read
      if (q + i + R::STAGES - 1 < n) next_tokens();
      cp_async_commit();
      multiply<T, MT, NT, PER>(tile[i], w4_smem + slot * R::BYTES, pieces, sum);
      slot = slot + 1 == R::STAGES ? 0 : slot + 1;
      if (q + i + AHEAD < n) next_weights(i);
      if (++kt == ct && a.splits == 1) {
        kt = 0;
#pragma unroll
        for (int mt = 0; mt < (GATED ? 1 : MT); ++mt)
          each(now, mt, [&](int r, int tok, float v, float w) { finish(now, now.rt + mt, r, tok, v, w); });
        clear();
        if (++i0 < i1) now = item_at(i0);
      }
    }
  }
  if (a.splits == 1) return;

  // the cluster's blocks' sums, in the order of their parts of K
  cp_async_wait<0>();
  __syncthreads();
  constexpr int LD = WARPS * MT * TILE_ROWS + 8;
  float* sums = reinterpret_cast<float*>(w4_smem);  // [token][warp, tile, row]
#pragma unroll
  for (int mt = 0; mt < (GATED ? 1 : MT); ++mt)
    each(now, mt, [&](int r, int tok, float v, float w) {
      sums[tok * LD + (warp * MT + mt) * TILE_ROWS + r] = v;
      if (GATED) sums[tok * LD + (warp * MT + 1) * TILE_ROWS + r] = w;
    });
  cluster_sync();
  constexpr int ROWS = GROUP * TILE_ROWS;
  for (int i = threadIdx.x + THREADS * sp; i < now.count * ROWS; i += THREADS * a.splits) {
    const int tok = i / ROWS, r = i % ROWS, at = tok * LD + (GATED ? r / TILE_ROWS * 2 * TILE_ROWS + r % TILE_ROWS : r);
    float v = 0.0f, w = 0.0f;
    for (int k = 0; k < a.splits; ++k) {
      v += ld_cluster(sums + at, k);
      if (GATED) w += ld_cluster(sums + at + TILE_ROWS, k);
    }
    finish(now, now.rt - (GATED ? warp : warp * MT) + r / TILE_ROWS, r % TILE_ROWS, tok, v, w);
  }
  cluster_sync();  // no block leaves while another may read its sums
}

template <int MT, int NT>
constexpr int rows_smem() {
  const int sums = 8 * NT * (WARPS * MT * TILE_ROWS + 8) * 4;
  return Ring<NT>::TOTAL > sums ? Ring<NT>::TOTAL : sums;
}

// Blocks of a launch: an item a cluster, or as many as share the items evenly.  Two blocks an SM.
struct RowsPlan {
  int splits;
  unsigned grid;
};
inline RowsPlan plan_rows(int64_t items, int ct) {
  RowsPlan p = {1, 0};
  const int64_t most = 2ll * device_sms();
  while (p.splits < 8 && items * p.splits * 2 <= most && ct >= 4 * p.splits) p.splits *= 2;
  if (p.splits > 1) {
    p.grid = (unsigned)(items * p.splits);
  } else {
    const int64_t run = (items + most - 1) / most;
    p.grid = (unsigned)((items + run - 1) / run);
  }
  return p;
}

template <typename T, int MT, int NT, int PER, int PARTS, bool GATED, int HPARTS, int AHEAD>
fgq_status launch_rows(const RowsArgs& a, unsigned grid, bool chained, cudaStream_t s) {
  constexpr auto kernel = rows_kernel<T, MT, NT, PER, PARTS, GATED, HPARTS, AHEAD>;
  constexpr int smem = rows_smem<MT, NT>();
  if (!tc::smem_attr_once<rows_kernel<T, MT, NT, PER, PARTS, GATED, HPARTS, AHEAD>>(smem)) return FGQ_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  unsigned n = 0;
  if (chained) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (a.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)a.splits;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return after_launch(cudaLaunchKernelEx(&cfg, kernel, a));
}

}  // namespace w4
}  // namespace fgq
