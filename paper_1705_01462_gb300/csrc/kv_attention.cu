// Attention over the 4-bit cache: the C entry, the choice of kernel and of the split, and the kernel
// that joins the chunks of a split.
#include "kv_attention.cuh"

namespace fgq {
namespace {

using namespace dec;

constexpr int JOIN_THREADS = 512;
constexpr uint64_t AT_TIMEOUT_NS = 1000000000ull;  // 1 s per wait

// out[row] = sum_c 2^(r_c - r) part_c / sum_c 2^(r_c - r) l_c over the chunks that had work; one block per row,
// JOIN_THREADS / D chunks at a time, each thread keeping the largest r so far (one pass, no load waits for
// another).  What precedes the wait reads only what was there before the attention kernel.
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const __grid_constant__ AttnArgs a, int tile_rows) {
  constexpr int WAYS = JOIN_THREADS / D, AHEAD = 8;
  __shared__ float sv[WAYS][D], sr[WAYS], sl[WAYS];
  const int64_t orow = blockIdx.x;  // (b, query, head)
  const int hq = (int)(orow % a.q_heads);
  const int64_t bt = orow / a.q_heads;
  const int qi = (int)(bt % a.T), b = (int)(bt / a.T);
  const int tid = threadIdx.x, d = tid % D, way = tid / D;
  const int n = seq_len(a, b);
  const int nq = a.q_lens ? min(__ldg(a.q_lens + b), a.T) : a.T;
  const int r0 = (qi * a.group + hq % a.group) / tile_rows * tile_rows;  // the block's tile of query rows
  int first, end;
  visible(a, n, nq, r0 / a.group, (min(r0 + tile_rows, a.rows) - 1) / a.group, first, end);
  first &= ~15;
  const int chunks = (int)min((int64_t)a.chunks, ((int64_t)end - first + a.chunk - 1) / a.chunk);
  const float2* st = reinterpret_cast<const float2*>(a.stats) + orow * a.chunks;
  const float* part = a.part + orow * a.chunks * D + d;
  pdl_wait();
  float r = AT_M0, v = 0.0f, l = 0.0f;
  for (int c0 = way; c0 < chunks; c0 += WAYS * AHEAD) {
    float2 s[AHEAD];
    float x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int c = c0 + i * WAYS;
      s[i] = c < chunks ? st[c] : make_float2(AT_M0, 0.0f);
      x[i] = c < chunks ? part[(int64_t)c * D] : 0.0f;
    }
    float top = r;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, s[i].x);
    const float f0 = ex2(r - top);
    v *= f0;
    l *= f0;
    r = top;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const float f = ex2(s[i].x - r);
      l = fmaf(f, s[i].y, l);
      v = fmaf(f, x[i], v);
    }
  }
  sv[way][d] = v;
  if (d == 0) {
    sr[way] = r;
    sl[way] = l;
  }
  __syncthreads();
  if (way == 0) {
    float top = AT_M0;
#pragma unroll
    for (int i = 0; i < WAYS; ++i) top = fmaxf(top, sr[i]);
    v = l = 0.0f;
#pragma unroll
    for (int i = 0; i < WAYS; ++i) {
      const float f = ex2(sr[i] - top);
      v = fmaf(f, sv[i][d], v);
      l = fmaf(f, sl[i], l);
    }
    store_out(a, orow * D + d, normalise(v, l));
  }
}

}  // namespace

constexpr int PROMPT_MIN_ROWS = 33;

fgq_status launch_attention_call(const fgq_kv_cache* cache, AttnArgs a, int max_len, cudaStream_t s) {
  const int D = cache->head_dim, nb = D / 32, gb = cache->group / 32;
  const bool split = a.type == FGQ_F32;
  const AttnKernel k = !split && a.rows >= PROMPT_MIN_ROWS ? prompt_kernel(D, cache->group, a.rows)
                       : nb == 2   ? attention_kernel_2(gb, split, a.rows)
                       : nb == 4 ? attention_kernel_4(gb, split, a.rows)
                                 : attention_kernel_8(gb, split, a.rows);
  a.row_tiles = (a.rows + k.rows - 1) / k.rows;
  const int64_t units = (int64_t)a.B * a.c.kv_heads * a.row_tiles;
  int64_t span = max_len;  // tokens that one block may have to read
  if (a.window && (int64_t)a.window + k.rows / a.group + 1 < span) span = (int64_t)a.window + k.rows / a.group + 1;
  span += 15;
  // the split: whole waves of blocks, as many as cost least if every sequence is as long as the longest may
  // be, a block costing its tokens and about 256 more; 128 tokens at least
  const int64_t slots = (int64_t)device_sms() * k.per_sm;
  int64_t chunk = 0, best = INT64_MAX;
  for (int waves = 1; waves <= 8; ++waves) {
    const int64_t n = waves * slots / units > 0 ? waves * slots / units : 1;
    const int64_t r = (span + n - 1) / n, c = r > 512 ? (r + 255) / 256 * 256 : (r + 127) / 128 * 128;
    const int64_t blocks = units * ((span + c - 1) / c), cost = (blocks + slots - 1) / slots * (c + 256);
    if (cost < best) {
      best = cost;
      chunk = c;
    }
  }
  a.chunk = (int)chunk;
  a.chunks = (int)((span + chunk - 1) / chunk);
  if (units * a.chunks > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  // few chunks that all run at once join as a cluster: no temporary and no second launch.  More blocks than
  // that would wait for eight of them to fit together.
  a.cluster = k.clusters && a.chunks > 1 && a.chunks <= 8 && units * a.chunks <= slots;
  const bool join = a.chunks > 1 && !a.cluster;
  void* tmp = nullptr;
  const int64_t orows = (int64_t)a.B * a.T * a.q_heads;
  if (join) {
    tmp = scratch_alloc((size_t)orows * a.chunks * (D + 2) * 4, s);
    if (!tmp) return FGQ_ERR_CUDA;
    a.part = static_cast<float*>(tmp);
    a.stats = a.part + (size_t)orows * a.chunks * D;
  }
  fgq_status st = k.launch(a, (unsigned)(units * a.chunks), s);
  if (st == FGQ_OK && join) {
    const dim3 grid((unsigned)orows), block(JOIN_THREADS);
    st = after_launch(D == 64    ? launch_pdl(join_kernel<64>, grid, block, 0, s, a, k.rows)
                      : D == 128 ? launch_pdl(join_kernel<128>, grid, block, 0, s, a, k.rows)
                                 : launch_pdl(join_kernel<256>, grid, block, 0, s, a, k.rows));
  }
  if (tmp && cudaFreeAsync(tmp, s) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

}  // namespace fgq

using namespace fgq;

extern "C" fgq_status fgq_kv_attention(const fgq_kv_cache* cache, const void* q, fgq_float_type type, int B, int T,
                                       int q_heads, int64_t q_batch_stride, int64_t q_token_stride,
                                       const int32_t* page_table, int max_pages, const int32_t* seq_lens,
                                       const int32_t* q_lens, int max_len, int causal, int window, float scale,
                                       void* out, cudaStream_t stream) {
  if (B < 0 || T < 0 || q_heads <= 0 || max_pages < 0 || max_len < 0 || window < 0 || !dec::valid_float(type))
    return FGQ_ERR_ARG;
  if ((causal != 0 && causal != 1) || (window && !causal) || !(scale > 0.0f) || dec::nonfinite_host(scale))
    return FGQ_ERR_ARG;
  const fgq_status st = dec::check_cache(cache);
  if (st != FGQ_OK) return st;
  if (q_heads % cache->kv_heads != 0) return FGQ_ERR_ARG;
  if (B == 0 || T == 0) return FGQ_OK;
  if (!q || !out || !page_table || !seq_lens) return FGQ_ERR_ARG;
  if (!dec::aligned(q, 16) || !dec::aligned(out, 16) || !dec::aligned(page_table, 4) || !dec::aligned(seq_lens, 4) ||
      !dec::aligned(q_lens, 4) || !dec::stride16(q_batch_stride, type) || !dec::stride16(q_token_stride, type))
    return FGQ_ERR_ALIGN;
  const int group = q_heads / cache->kv_heads;
  const int64_t capacity = (int64_t)max_pages * cache->page_size;
  if ((int64_t)T * group > INT32_MAX / 2 || (int64_t)B * T * q_heads > INT32_MAX || capacity > INT32_MAX)
    return FGQ_ERR_UNSUPPORTED;
  dec::AttnArgs a = {};
  a.c = dec::view(cache, page_table, max_pages);
  a.q = q;
  a.out = out;
  a.qbs = q_batch_stride;
  a.qts = q_token_stride;
  a.seq_lens = seq_lens;
  a.q_lens = q_lens;
  a.err = device_error_word();
  const int64_t lim_us = debug_wait_limit_us();
  a.timeout_ns = lim_us < 0 ? AT_TIMEOUT_NS : (uint64_t)lim_us * 1000u;
  a.scale_log2 = scale * 1.44269504f;
  a.type = type;
  a.B = B;
  a.T = T;
  a.q_heads = q_heads;
  a.group = group;
  a.rows = T * group;
  a.causal = causal;
  a.window = window;
  const int bound = max_len > 0 && max_len < capacity ? max_len : (int)(capacity > 0 ? capacity : 1);
  return launch_attention_call(cache, a, bound, stream);
}
