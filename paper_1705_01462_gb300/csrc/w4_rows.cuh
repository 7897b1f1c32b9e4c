// The product of few tokens with 4-bit weights, tokens in a ring that a block's eight warps share: for small matrices, and where tokens are
// too many or too long to be held (w4_resident.cuh).  A small matrix is bound by the way to its first products and a cluster's join: 8
// tokens of bf16, 4096 -> 4096, 6.0 us, 1.3 of them bytes; 1024 -> 2048 4.2.  A large one by the shared-memory reads of 16 or 32 columns, which
// each warp makes for 16 rows of weights: 16 tokens, 8192 -> 131072, 192 us for 84.5 of bytes.
#pragma once

#include "linear_internal.cuh"
#include "w4.cuh"

namespace fgq {
namespace w4 {

struct RowsArgs {
  Matrix w;
  TokenRows x;
  int splits;  // blocks of a cluster that share K
  // items (rows, tokens), the tokens' tiles first
  const float* bias;
  void* y;
  int P, M, ytype, items, token_tiles;
  int early;  // the kernel before is this library's: weights may be loaded while it runs
};

// RAW: tokens go through registers.
template <typename T, int NT, int PER, int PARTS, int AHEAD, bool RAW>
__global__ void __launch_bounds__(THREADS, 2) rows_kernel(const __grid_constant__ RowsArgs a) {
  using R = Ring<NT>;
  constexpr int CPT = columns_per_token(PARTS), TOKENS = 8 * NT / CPT;
  extern __shared__ __align__(16) uint8_t w4_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int items = a.items;
  int sp = 0, i0, i1;
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
    int64_t first;        // its first tile's number for this warp; a row tile past the last is read as the last
    int rt, tok0, count;  // row tile of this warp, first token, how many there are
  };
  auto item_at = [&](int i) {
    Item it;
    const int rg = i / a.token_tiles, tt = i - rg * a.token_tiles;
    it.rt = rg * WARPS + warp;
    it.first = (int64_t)min(it.rt, a.w.rt - 1) * a.w.ct + c0;
    it.tok0 = tt * TOKENS;
    it.count = min(TOKENS, a.P - it.tok0);
    return it;
  };
  Tile<PER> tile[AHEAD][1];
  Columns<NT> cols;
  auto columns = [&](const Item& it) {
#pragma unroll
    for (int i = 0; i < R::COPIES; ++i) {
      const int tok = (int)(threadIdx.x >> 4) + 16 * i;
      cols.off[i] = -1;
      if (tok < it.count) {
        cols.off[i] = 2 * ((it.tok0 + tok) * a.x.pitch);
      }
    }
  };

  const uint8_t* xb = static_cast<const uint8_t*>(a.x.data);
  const uint32_t ring_at = smem_u32(w4_smem);
  // three places in the sequence of stages: the weights to load, the tokens to copy, and the stage to multiply
  Item now = item_at(i0), wit = now, xit = now;
  int kt = 0, wi = i0, wkt = 0, xi = i0, xkt = 0, xslot = 0, slot = 0;
  auto next_weights = [&](int at) {
    tile[at][0].load(a.w.codes, a.w.scales, wit.first + wkt, lane);
    if (++wkt == ct) {
      wkt = 0;
      if (++wi < i1) wit = item_at(wi);
    }
  };
  auto next_place = [&]() {
    if (++xkt == ct) {
      xkt = 0;
      if (++xi < i1) {
        xit = item_at(xi);
        if (!RAW) columns(xit);
      }
    }
  };
  auto next_slot = [&]() { xslot = xslot + 1 == R::STAGES ? 0 : xslot + 1; };
  auto next_tokens = [&]() {
    cols.copy(ring_at + xslot * R::BYTES, xb, c0 + xkt, a.x.kvalid);
    next_slot();
    next_place();
  };
  // tokens that go through registers: loaded a stage before they are stored
  constexpr int PIECES = (TOKENS + 15) / 16;  // of a thread and stage
  const int chunk = threadIdx.x & 15;
  auto fetch = [&](Eight<PARTS>(&e)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int tok = (int)(threadIdx.x >> 4) + 16 * i;
      e[i].load(a.x, tok < xit.count ? xit.tok0 + tok : -1, (c0 + xkt) * TILE_COLS + 8 * chunk);
    }
    next_place();
  };
  auto put = [&](const Eight<PARTS>(&e)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int tok = (int)(threadIdx.x >> 4) + 16 * i;
      if (tok < TOKENS) e[i].store(w4_smem + xslot * R::BYTES, tok, chunk);
    }
    next_slot();
  };
  Eight<PARTS> ahead[PIECES];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < n) next_weights(i);
  if (a.early) pdl_wait();
  if constexpr (!RAW) {
    columns(xit);
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i) {
      if (i < n) next_tokens();
      cp_async_commit();
    }
  } else {
    Eight<PARTS> first[R::STAGES - 1][PIECES];
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i)
      if (i < n) fetch(first[i]);
    if (R::STAGES - 1 < n) fetch(ahead);
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i)
      if (i < n) put(first[i]);
  }
  pair_t sum[1][NT][2];
  auto clear = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sum[0][nt][0] = sum[0][nt][1] = 0ull;
  };
  clear();

  // what becomes of a finished sum: of row r of the item's first row tile `rt`, and of token tok
  auto finish = [&](const Item& it, int rt, int r, int tok, float v) {
    const int m = rt * TILE_ROWS + r;
    if (m < a.M)
      store_typed(a.y, a.ytype, (int64_t)(it.tok0 + tok) * a.M + m, fmaf(v, Operand<T>::BACK, a.bias ? __ldg(a.bias + m) : 0.0f));
  };
  // this lane's sums as those of tokens: value (row g or g + 8) of token `tok`, or none
  auto each = [&](const Item& it, auto f) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float s[2];
        unpack_f2(sum[0][nt][half], s[0], s[1]);
        if constexpr (CPT == 1) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (8 * nt + 2 * t + e < it.count) f(g + 8 * half, 8 * nt + 2 * t + e, s[e]);
        } else {  // three parts, and a column that is zero
          float v = s[0] + s[1];
          v += __shfl_xor_sync(FULL_MASK, v, 1);
          const int tok = 2 * nt + (t >> 1);
          if ((t & 1) == 0 && tok < it.count) f(g + 8 * half, tok, v);
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
      if constexpr (!RAW) {
        if (q + i + R::STAGES - 1 < n) next_tokens();
        cp_async_commit();
      } else if (q + i + R::STAGES - 1 < n) {
        put(ahead);
        if (q + i + R::STAGES < n) fetch(ahead);
      }
      multiply<T, 1, NT, PER>(tile[i], w4_smem + slot * R::BYTES, pieces, sum);
      slot = slot + 1 == R::STAGES ? 0 : slot + 1;
      if (q + i + AHEAD < n) next_weights(i);
      if (++kt == ct && a.splits == 1) {
        kt = 0;
        each(now, [&](int r, int tok, float v) { finish(now, now.rt, r, tok, v); });
        clear();
        if (++i0 < i1) now = item_at(i0);
      }
    }
  }
  if (a.splits == 1) return;

  // the cluster's blocks' sums, in the order of their parts of K
  cp_async_wait<0>();
  __syncthreads();
  constexpr int ROWS = WARPS * TILE_ROWS, LD = ROWS + 8;
  float* sums = reinterpret_cast<float*>(w4_smem);  // [token][warp, row]
  each(now, [&](int r, int tok, float v) { sums[tok * LD + warp * TILE_ROWS + r] = v; });
  cluster_sync();
  for (int i = threadIdx.x + THREADS * sp; i < now.count * ROWS; i += THREADS * a.splits) {
    const int tok = i / ROWS, r = i % ROWS;
    float v = 0.0f;
    for (int k = 0; k < a.splits; ++k) v += ld_cluster(sums + tok * LD + r, k);
    finish(now, now.rt - warp, r, tok, v);
  }
  cluster_sync();  // no block leaves while another may read its sums
}

template <int NT>
constexpr int rows_smem() {
  const int sums = 8 * NT * (WARPS * TILE_ROWS + 8) * 4;
  return Ring<NT>::TOTAL > sums ? Ring<NT>::TOTAL : sums;
}

// Blocks of a launch: an item a cluster.  Rows of four tile columns and more are split, down to one or two a block where that is one block an SM
// at most (bf16, 32 tokens, 1024 -> 2048 5.6 us, four columns at least 6.4; but 256 -> 256 6.2 and not split 4.6), and to two or more where it is
// two (fp32, 32 tokens, 1111 -> 999 6.9, one or two 8.5; bf16, 64 tokens, 2048 -> 4096 9.5, eight or more 11.1).  Or as many as share the items
// evenly, two an SM.
struct RowsPlan {
  int splits;
  unsigned grid;
};
inline RowsPlan plan_rows(int64_t items, int ct) {
  RowsPlan p = {1, 0};
  const int64_t sms = device_sms(), most = 2 * sms;
  while (p.splits < 8 && ct >= 4 && ct >= 2 * p.splits) {
    const int64_t blocks = items * p.splits * 2;
    if (blocks > most || (blocks > sms && ct < 4 * p.splits)) break;
    p.splits *= 2;
  }
  if (p.splits > 1) {
    p.grid = (unsigned)(items * p.splits);
  } else {
    const int64_t run = (items + most - 1) / most;
    p.grid = (unsigned)((items + run - 1) / run);
  }
  return p;
}

template <typename T, int NT, int PER, int PARTS, int AHEAD, bool RAW>
fgq_status launch_rows(const RowsArgs& a, unsigned grid, bool chained, cudaStream_t s) {
  constexpr auto kernel = rows_kernel<T, NT, PER, PARTS, AHEAD, RAW>;
  constexpr int smem = rows_smem<NT>();
  if (!tc::smem_attr_once<rows_kernel<T, NT, PER, PARTS, AHEAD, RAW>>(smem)) return FGQ_ERR_CUDA;
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
