// Attention over the 4-bit cache: the C entry, the choice of kernel and of the split, and the kernel
// that joins the chunks of a split.
#include "kv_attention.cuh"

namespace fgq {
namespace {

using namespace dec;

constexpr int JOIN_THREADS = 512, JOIN_FEW = 16;
constexpr uint64_t AT_TIMEOUT_NS = 1000000000ull;  // 1 s per wait

// The chunks of output row orow = (b, query, head) that had work.
__device__ __forceinline__ int chunks_of(const AttnArgs& a, int64_t orow, int tile_rows) {
  const int hq = (int)(orow % a.q_heads);
  const int64_t bt = orow / a.q_heads;
  const int qi = (int)(bt % a.T), b = (int)(bt / a.T);
  const int n = seq_len(a, b);
  const int nq = a.q_lens ? min(__ldg(a.q_lens + b), a.T) : a.T;
  const int r0 = (qi * a.group + hq % a.group) / tile_rows * tile_rows;  // the block's tile of query rows
  int first, end;
  visible(a, n, nq, r0 / a.group, (min(r0 + tile_rows, a.rows) - 1) / a.group, first, end);
  first &= ~15;
  return (int)min((int64_t)a.chunks, ((int64_t)end - first + a.chunk - 1) / a.chunk);
}

// The join where there are at most JOIN_FEW chunks: D / 4 threads a row, four values each, one chunk after
// another.  With few chunks there are many rows, and a block a row costs its start: 300 queries of 32 heads over
// 20000 tokens took 223 us with join_kernel throughout and 181 us with this one.  A long row is slow here, as one
// thread reads all its chunks: one query of 64 heads over 131071 tokens took 50 us instead of 43.
template <int D>
__global__ void __launch_bounds__(256) join_few_kernel(const __grid_constant__ AttnArgs a, int tile_rows, int64_t orows) {
  const int64_t orow = (int64_t)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  if (orow >= orows) return;  // no barrier, and no wait needed
  const int d = threadIdx.x % (D / 4) * 4;
  const int chunks = chunks_of(a, orow, tile_rows);
  const float2* st = reinterpret_cast<const float2*>(a.stats) + orow * a.chunks;
  const float* part = a.part + orow * a.chunks * D + d;
  pdl_wait();
  float r = AT_M0, l = 0.0f;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int c = 0; c < chunks; ++c) {
    const float2 s = st[c];
    const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)c * D);
    const float top = fmaxf(r, s.x), f0 = ex2(r - top), f = ex2(s.x - top);
    r = top;
    l = fmaf(f, s.y, l * f0);
    v.x = fmaf(f, x.x, v.x * f0);
    v.y = fmaf(f, x.y, v.y * f0);
    v.z = fmaf(f, x.z, v.z * f0);
    v.w = fmaf(f, x.w, v.w * f0);
  }
  const int64_t at = orow * D + d;
  store_out(a, at, normalise(v.x, l));
  store_out(a, at + 1, normalise(v.y, l));
  store_out(a, at + 2, normalise(v.z, l));
  store_out(a, at + 3, normalise(v.w, l));
}

// out[row] = sum_c 2^(r_c - r) part_c / sum_c 2^(r_c - r) l_c over the chunks that had work; one block per row,
// JOIN_THREADS / D chunks at a time, each thread keeping the largest r so far (one pass, no load waits for
// another).  What precedes the wait reads only what was there before the attention kernel.
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const __grid_constant__ AttnArgs a, int tile_rows) {
  constexpr int WAYS = JOIN_THREADS / D, AHEAD = 8;
  __shared__ float sv[WAYS][D], sr[WAYS], sl[WAYS];
  const int64_t orow = blockIdx.x;  // (b, query, head)
  const int tid = threadIdx.x, d = tid % D, way = tid / D;
  const int chunks = chunks_of(a, orow, tile_rows);
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

namespace {

// How a call could run: a kernel, its chunks of the longest sequence, and the time that takes if every
// sequence is as long.
struct Plan {
  AttnKernel k;
  int64_t units, chunks, chunk;
  float us;
  bool cluster;
};

// Whole waves of blocks, as many as cost least: the kernel's start, each further wave's, the tokens of the blocks that
// follow one another on an SM, and for a join kernel 3 us and the partial sums' way to memory and back.  (One token,
// 16 sequences of 16384 tokens, 8 kv heads of 128 values: 80 us in one or two waves, 90 in eight; 32 of 3000: 35 us in
// one, 41 in two; 40 of 1000 to 8000, 4 kv heads: 51 us in one, 41 in two.)
Plan plan_kernel(const AttnKernel& k, const AttnArgs& a, int D, int max_len) {
  Plan best = {};
  best.k = k;
  best.units = (int64_t)a.B * a.c.kv_heads * ((a.rows + k.rows - 1) / k.rows);
  int64_t span = max_len;  // tokens that one block may have to read
  if (a.window) {  // and from the start of a block of 16
    if ((int64_t)a.window + k.rows / a.group + 1 < span) span = (int64_t)a.window + k.rows / a.group + 1;
    span += 15;
  }
  const int64_t sms = device_sms(), slots = sms * k.per_sm;
  for (int waves = 1; waves <= 8; ++waves) {
    const int64_t want = waves * slots / best.units, n = want > 0 ? want : 1, r = (span + n - 1) / n;
    const int64_t step = k.clusters && r > 512 ? 256 : 128;  // a tile for each warp; for the prompt kernel's block
    const int64_t chunk = (r + step - 1) / step * step;
    const int64_t chunks = (span + chunk - 1) / chunk, blocks = best.units * chunks;
    // few chunks that all run at once join as a cluster: no temporary and no second launch.  More blocks than that
    // would wait for eight of them to fit together.  Each of the GPU's eight groups of SMs, which a cluster does
    // not cross, may leave chunks - 1 places empty: 24 rows of 256 values over 2 sequences of 20000 tokens, 288
    // blocks in clusters of 6 on 304 places, took 119 us, and 74 as separate blocks.
    const bool cluster = k.clusters && chunks > 1 && chunks <= 8 && blocks + 8 * (chunks - 1) <= slots;
    const int64_t full = blocks / slots, rest = blocks % slots, more = (blocks - 1) / slots;
    // the last blocks share an SM with fewer others, and run up to twice as fast as three together would
    const int64_t beside = rest ? (rest + sms - 1) / sms : 0, least = k.per_sm < 2 ? k.per_sm : 2;
    const float last = rest ? (float)(beside > least ? beside : least) / (float)k.per_sm : 0.0f;
    // and a twelfth of a chunk, as sequences are seldom all as long and shorter chunks even them out
    float us = k.start_us + (float)more * k.wave_us + ((float)full + last + 0.08f) * (float)chunk / k.rate;
    if (chunks > 1 && !cluster) us += 3.0f + (float)a.B * a.T * a.q_heads * chunks * D * 8.0f / 4e6f;
    if (waves == 1 || us < best.us) {
      best.chunk = chunk;
      best.chunks = chunks;
      best.us = us;
      best.cluster = cluster;
    }
  }
  return best;
}

}  // namespace

fgq_status launch_attention_call(const fgq_kv_cache* cache, AttnArgs a, int max_len, cudaStream_t s) {
  const int D = cache->head_dim, nb = D / 32, gb = cache->group / 32;
  Plan p = plan_kernel(nb == 2   ? attention_kernel_2(gb, a.type == FGQ_F32, a.rows)
                       : nb == 4 ? attention_kernel_4(gb, a.type == FGQ_F32, a.rows)
                                 : attention_kernel_8(gb, a.type == FGQ_F32, a.rows),
                       a, D, max_len);
  // From nine rows on, the prompt kernel may be faster: it dequantizes a tile of the cache once for 128 or 256 rows,
  // but its block takes an SM to itself and longer to start.  With heads of 128 values, 32 sequences of 2000 tokens
  // and 8 kv heads, 16 rows take 33 us here and 61 there, 64 rows 113 and 62; with 8 sequences of 4096 and 4 heads,
  // 12 rows 19 and 23, 64 rows 37 and 25; with 256 values 24 rows 39 and 35; with one sequence of 1000 and 64 values,
  // 64 rows 10.4 and 12.5.  So the estimates decide, and not the number of rows.
  const int only = debug_attention_kernel();
  if (a.type != FGQ_F32 && only != 1 && (a.rows > 8 || only == 2)) {
    AttnKernel k = prompt_kernel(D, cache->group, a.rows);
    if (a.type == FGQ_F16) k.rate *= 0.85f;  // a second product with the values
    const Plan q = plan_kernel(k, a, D, max_len);
    if (q.us < p.us || only == 2) p = q;
  }
  a.row_tiles = (a.rows + p.k.rows - 1) / p.k.rows;
  if (p.units * p.chunks > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  a.chunk = (int)p.chunk;
  a.chunks = (int)p.chunks;
  a.cluster = p.cluster;
  const bool join = a.chunks > 1 && !a.cluster;
  void* tmp = nullptr;
  const int64_t orows = (int64_t)a.B * a.T * a.q_heads;
  if (join) {
    tmp = scratch_alloc((size_t)orows * a.chunks * (D + 2) * 4, s);
    if (!tmp) return FGQ_ERR_CUDA;
    a.part = static_cast<float*>(tmp);
    a.stats = a.part + (size_t)orows * a.chunks * D;
  }
  fgq_status st = p.k.launch(a, (unsigned)(p.units * p.chunks), s);
  if (st == FGQ_OK && join && a.chunks <= JOIN_FEW) {
    const int rows = 256 / (D / 4);
    const dim3 grid((unsigned)((orows + rows - 1) / rows)), block(256);
    st = after_launch(D == 64    ? launch_pdl(join_few_kernel<64>, grid, block, 0, s, a, p.k.rows, orows)
                      : D == 128 ? launch_pdl(join_few_kernel<128>, grid, block, 0, s, a, p.k.rows, orows)
                                 : launch_pdl(join_few_kernel<256>, grid, block, 0, s, a, p.k.rows, orows));
  } else if (st == FGQ_OK && join) {
    const dim3 grid((unsigned)orows), block(JOIN_THREADS);
    st = after_launch(D == 64    ? launch_pdl(join_kernel<64>, grid, block, 0, s, a, p.k.rows)
                      : D == 128 ? launch_pdl(join_kernel<128>, grid, block, 0, s, a, p.k.rows)
                                 : launch_pdl(join_kernel<256>, grid, block, 0, s, a, p.k.rows));
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
