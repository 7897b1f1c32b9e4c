// The 4-bit cache of keys and values: quantization as it is written, and its read-back.
//
// Per group of G values of one token and head: lo = min rounded down to bf16, s = (max - lo) / 15
// rounded up to bf16, codes round((x - lo) / s).  Eight consecutive values, a 16-byte load of 16-bit
// elements, make one 32-bit word of a key row, or two 16-bit units of a value row; the G / 8 threads of
// a group find its extremes by shuffles.  Both kernels move each byte once; consecutive threads take consecutive
// values of the dense side, and the 32 to 128 bytes of a cache row are written by neighbouring threads, so that
// L2 merges them into whole sectors.
// 4 x 8192 tokens, 8 heads of 128 values, bf16, groups of 64, 174 MB each: appending 53 us, half the copy rate, as 22
// instructions a value (about three of them the quotient's) keep the issue slots 76% busy (ALU pipe 59%); read-back 41 us, 16
// instructions a value, issue slots 75% busy (ALU pipe 66%).
#include <type_traits>

#include "decoder_internal.cuh"

namespace fgq {
namespace {

using namespace dec;

constexpr int KV_THREADS = 256;

struct KvArgs {
  CacheView c;
  const void* k;
  const void* v;
  void* k_out;
  void* v_out;
  int64_t bs[2], ts[2];  // batch and token strides of k and v, in elements
  const int32_t* starts;
  const int32_t* lens;  // or nullptr
  int B, T;
  unsigned int* err;
};

// bf16 values next to x, as fp32: at or below it, and (x >= 0) at or above it.
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float(((u & 0x80000000u) ? u + 0xffffu : u) & 0xffff0000u);
}
__device__ __forceinline__ float bf16_up_pos(float x) {
  return __uint_as_float((__float_as_uint(x) + 0xffffu) & 0xffff0000u);
}

// What both kernels share: a warp takes a run of RUN = KV_TOKENS (256 / D) consecutive tokens of one head, so
// that it writes whole 128-byte lines of the cache (two heads' 64 bytes side by side filled the path to L2 with
// small requests: 92 us for 4 x 8192 tokens, 8 heads of 128); warps count (run, head), heads fastest.
// blockIdx.y: sequences (strided); blockIdx.z: keys, values.  Of KV_TOKENS rows a thread has values
// 8 u .. 8 u + 7: as many loads under way.
constexpr int KV_TOKENS = 4;
template <int D>
struct KvRun {
  static constexpr int LR = D / 8, ROWS = 32 / LR, RUN = ROWS * KV_TOKENS;  // lanes of a row, rows of a warp at once
};

// Cache rows of a run of at most 16 positions from pos on, `live` of which are wanted: they span two pages at most.
struct RowRun {
  int64_t first, second;  // row of the first position; of the first one in the next page; -1: none there
  int in_first, live;     // positions in the first page
  __device__ __forceinline__ RowRun(const CacheView& c, int b, int head, int64_t pos, int live_) : live(live_) {
    first = second = -1;
    in_first = 0;
    if (live <= 0) return;
    first = cache_row(c, b, head, pos);
    const int slot = pos >= 0 ? (int)((uint32_t)pos - page_of(c, (uint32_t)pos) * (uint32_t)c.page_size)
                              : c.page_size - (int)min((int64_t)16, -pos);  // the positions before 0 are nowhere
    in_first = c.page_size - slot;
    if (in_first < live) second = cache_row(c, b, head, pos + in_first);
  }
  __device__ __forceinline__ bool whole(int n) const { return live >= n && in_first >= n && first >= 0; }
  __device__ __forceinline__ int64_t at(int i) const {
    if (i >= live) return -1;
    return i < in_first ? (first < 0 ? -1 : first + i) : (second < 0 ? -1 : second + (i - in_first));
  }
};

// Extremes of a group from its GL threads' (NaN where one holds NaN); 16-bit types both in one word.
template <typename T, int GL>
__device__ __forceinline__ void group_extremes(float& lo, float& hi) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) {
      lo = min_nan(lo, __shfl_xor_sync(FULL_MASK, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(FULL_MASK, hi, o));
    }
  } else {
    uint32_t v = pack2(lo, -hi, T());
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) v = min2_nan(v, __shfl_xor_sync(FULL_MASK, v, o), T());
    const float2 f = unpack2(v, T());
    lo = f.x;
    hi = -f.y;
  }
}

// Four codes (plus kMagicI each) as 16 bits.
__device__ __forceinline__ uint32_t nibbles(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return a + 16u * b + 256u * c + 4096u * d - 4369u * (uint32_t)kMagicI;
}

// Groups that the common path leaves out: NaN or Inf (zeros, and bad), magnitudes above 2^126, whose differences
// may overflow where those of their halves do not, and ranges below 1e-25, constant groups among them.
__device__ __forceinline__ void quantize_rare(const float (&x)[8], float lo, float hi, float& l, float& s, uint32_t (&c)[8],
                                           bool& bad) {
  bad = nonfinite(lo) || nonfinite(hi);
  if (bad) lo = hi = 0.0f;
  const bool huge = fmaxf(fabsf(lo), fabsf(hi)) > 8.507059e37f;
  const float f = huge ? 0.5f : 1.0f;
  l = fmaxf(bf16_down(lo * f), huge ? -1.6947657e38f : -3.3895314e38f);
  s = bf16_up_pos(fmaxf(__fdiv_rn(hi * f - l, 15.0f), 0.0f));
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float q = s > 0.0f && !bad ? __fdiv_rn(x[k] * f - l, s) : 0.0f;
    c[k] = (uint32_t)kMagicI + (uint32_t)min(max((int)rintf(q), 0), 15);
  }
  if (huge) l *= 2.0f, s *= 2.0f;
}

// Words of a value row: unit (g, j) of 16 bits is the half j % 2 of word (g NB + j) / 2.  The thread of block j
// and quarter v has units (2 v, j) and (2 v + 1, j), its neighbour at j ^ 1 the words' other halves: each of the
// two takes one whole word.
__device__ __forceinline__ uint32_t swap_neighbour(uint32_t give) { return __shfl_xor_sync(FULL_MASK, give, 4); }

template <typename T, int D, int G>
__global__ void __launch_bounds__(KV_THREADS, 4) kv_append_kernel(const __grid_constant__ KvArgs a) {
  using R = KvRun<D>;
  constexpr int LR = R::LR, GL = G / 8, NB = D / 32, NG = D / G;
  const int of_v = blockIdx.z;
  const int lane = threadIdx.x & 31, u = lane % LR, sub = lane / LR;  // row of those the warp has at once
  const uint32_t r = blockIdx.x * (KV_THREADS / 32) + threadIdx.x / 32;  // below 2^32: the host checks
  const int t0 = (int)(r / (uint32_t)a.c.kv_heads) * R::RUN;
  const int head = (int)(r % (uint32_t)a.c.kv_heads);
  const int j = u >> 2, v = u & 3;  // block of 32, quarter of it
  const T* src = static_cast<const T*>(of_v ? a.v : a.k) + (int64_t)head * D + 8 * u;
  const int64_t bs = of_v ? a.bs[1] : a.bs[0], ts = of_v ? a.ts[1] : a.ts[0];
  uint32_t* codes = reinterpret_cast<uint32_t*>(of_v ? a.c.v_codes : a.c.k_codes);
  uint32_t* params = of_v ? a.c.v_params : a.c.k_params;
  const int at = of_v ? ((2 * v + (j & 1)) * NB + j) >> 1 : v * NB + j;  // this thread's word of a row
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int n = a.lens ? min(__ldg(a.lens + b), a.T) : a.T;
    if (t0 >= n) continue;  // the whole warp; its later rows may be past the end, their lanes take part in shuffles
    uint32_t par[KV_TOKENS];
    Raw8<T> raw[KV_TOKENS];
    const int64_t start = __ldg(a.starts + b);
#pragma unroll
    for (int i = 0; i < KV_TOKENS; ++i) {
      raw[i].zero();
      const int t = t0 + i * R::ROWS + sub;
      if (t < n) raw[i].load(src + b * bs + t * ts);
    }
    const RowRun rows(a.c, b, head, start + t0, n - t0);
    const bool whole = rows.whole(R::RUN);
    uint32_t* out = codes + (rows.first + sub) * (D / 8) + at;  // of a whole run
    bool any_bad = false;
#pragma unroll
    for (int i = 0; i < KV_TOKENS; ++i) {
      float lo, hi;
      raw[i].extremes(lo, hi);
      group_extremes<T, GL>(lo, hi);
      float x[8], l, s;
      raw[i].unpack(x);
      uint32_t c[8];  // the codes, each plus kMagicI (the integers of 1.5 2^23 + c)
      bool bad = false;
      const float d = hi - lo;
      if (fmaxf(fabsf(lo), fabsf(hi)) <= 8.507059e37f && d >= 1e-25f) {  // not for NaN
        l = bf16_down(lo);
        const float e = hi - l;
        // e / 15 correctly rounded: the product with RN(1 / 15) corrected by its exact remainder (Markstein)
        const float q0 = e * 0.0666666701f;
        s = bf16_up_pos(fmaf(fmaf(-15.0f, q0, e), 0.0666666701f, q0));
        // RN(1 / s): the approximation after one Newton step (s has 8 bits, 1 / s is far from a rounding
        // boundary), and with it the correctly rounded quotient, again by its exact remainder: of 24 by 8 bits,
        // no quotient lies within 2^-9 ulp of a boundary
        float y;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
        y = fmaf(fmaf(-s, y, 1.0f), y, y);
        const uint64_t l2 = pack_f2(-l, -l), y2 = pack_f2(y, y), ms2 = pack_f2(-s, -s), magic2 = pack_f2(kMagicF, kMagicF);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint64_t a = add_f2(pack_f2(x[2 * k], x[2 * k + 1]), l2), q = mul_f2(a, y2);
          float m0, m1;
          unpack_f2(add_f2(fma_f2(fma_f2(q, ms2, a), y2, q), magic2), m0, m1);  // rounds half to even
          c[2 * k] = __float_as_uint(m0);
          c[2 * k + 1] = __float_as_uint(m1);
        }
      } else {
        quantize_rare(x, lo, hi, l, s, c, bad);
      }
      uint32_t w;
      if (!of_v) {
        w = nibbles(c[0], c[2], c[4], c[6]) + (nibbles(c[1], c[3], c[5], c[7]) << 16);
      } else {
        const uint32_t first = nibbles(c[0], c[1], c[2], c[3]), second = nibbles(c[4], c[5], c[6], c[7]);
        const uint32_t got = swap_neighbour(j & 1 ? first : second);
        w = j & 1 ? got | second << 16 : first | got << 16;
      }
      par[i] = (__float_as_uint(l) & 0xffff0000u) | (__float_as_uint(s) >> 16);
      any_bad |= bad && t0 + i * R::ROWS + sub < n;
      if (whole) {
        out[i * R::ROWS * (D / 8)] = w;
      } else {
        const int64_t row = rows.at(i * R::ROWS + sub);
        if (t0 + i * R::ROWS + sub < n && row < 0) record_error(a.err, FGQ_ERR_ARG);
        if (row >= 0) codes[row * (D / 8) + at] = w;
      }
    }
    if (any_bad) record_error(a.err, FGQ_ERR_NONFINITE);
    // the run's parameters, one a lane (RUN NG <= 32 of them), in the order of the cache
    const int k = lane / NG, gi = lane % NG;
    uint32_t mine = 0u;
#pragma unroll
    for (int i = 0; i < KV_TOKENS; ++i) {
      const uint32_t got = __shfl_sync(FULL_MASK, par[i], k % R::ROWS * LR + gi * GL);
      if (k / R::ROWS == i) mine = got;
    }
    if (k < R::RUN) {
      const int64_t row = rows.at(k);
      if (row >= 0) params[row * NG + gi] = mine;
    }
  }
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(const __grid_constant__ KvArgs a) {
  using R = KvRun<D>;
  constexpr int LR = R::LR, GL = G / 8, NB = D / 32, NG = D / G;
  const int of_v = blockIdx.z;
  const int lane = threadIdx.x & 31, u = lane % LR, sub = lane / LR;  // row of those the warp has at once
  const uint32_t r = blockIdx.x * (KV_THREADS / 32) + threadIdx.x / 32;
  const int t0 = (int)(r / (uint32_t)a.c.kv_heads) * R::RUN;
  const int head = (int)(r % (uint32_t)a.c.kv_heads);
  const int j = u >> 2, v = u & 3;
  T* dst = static_cast<T*>(of_v ? a.v_out : a.k_out) + (int64_t)head * D + 8 * u;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(of_v ? a.c.v_codes : a.c.k_codes);
  const uint32_t* params = of_v ? a.c.v_params : a.c.k_params;
  const int at = of_v ? ((2 * v + (j & 1)) * NB + j) >> 1 : v * NB + j;
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int n = a.lens ? min(__ldg(a.lens + b), a.T) : a.T;
    const RowRun rows(a.c, b, head, (int64_t)__ldg(a.starts + b) + t0, n - t0);
    uint32_t w[KV_TOKENS], p[KV_TOKENS];
#pragma unroll
    for (int i = 0; i < KV_TOKENS; ++i) {
      w[i] = p[i] = 0u;  // code 0 of zero parameters: the value 0
      if (t0 + i * R::ROWS + sub < n) {
        const int64_t row = rows.at(i * R::ROWS + sub);
        if (row < 0) {
          record_error(a.err, FGQ_ERR_ARG);
        } else {
          w[i] = codes[row * (D / 8) + at];
          p[i] = params[row * NG + u / GL];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < KV_TOKENS; ++i) {
      const float lo = __uint_as_float(p[i] & 0xffff0000u), s = __uint_as_float(p[i] << 16);
      float x[8];
      if (!of_v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = fmaf(s, (float)(w[i] >> (4 * e) & 15u), lo);  // s c is exact in fp32
          x[2 * e + 1] = fmaf(s, (float)(w[i] >> (16 + 4 * e) & 15u), lo);
        }
      } else {
        const uint32_t got = swap_neighbour(w[i]);
        const uint32_t c = j & 1 ? __byte_perm(got, w[i], 0x7632) : __byte_perm(w[i], got, 0x5410);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(s, (float)(c >> (4 * e) & 15u), lo);
      }
      const int t = t0 + i * R::ROWS + sub;
      if (t < a.T) store8(dst + ((int64_t)b * a.T + t) * a.c.kv_heads * D, x);
    }
  }
}

template <typename T, int D, int G>
fgq_status launch_kv(const KvArgs& a, bool append, cudaStream_t s) {
  constexpr int RUN = KvRun<D>::RUN, WARPS = KV_THREADS / 32;
  const int64_t runs = ((int64_t)a.T + RUN - 1) / RUN * a.c.kv_heads, blocks = (runs + WARPS - 1) / WARPS;
  if (a.T > MAX_SIZE || (int64_t)a.T * a.c.kv_heads > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)(a.B < 65535 ? a.B : 65535), 2);
  if (append)
    kv_append_kernel<T, D, G><<<grid, KV_THREADS, 0, s>>>(a);
  else
    kv_read_kernel<T, D, G><<<grid, KV_THREADS, 0, s>>>(a);
  return after_launch();
}

template <typename T>
fgq_status launch_kv_t(const KvArgs& a, int D, int G, bool append, cudaStream_t s) {
  if (D == 64) return G == 32 ? launch_kv<T, 64, 32>(a, append, s) : launch_kv<T, 64, 64>(a, append, s);
  if (D == 128)
    return G == 32   ? launch_kv<T, 128, 32>(a, append, s)
           : G == 64 ? launch_kv<T, 128, 64>(a, append, s)
                     : launch_kv<T, 128, 128>(a, append, s);
  return G == 32   ? launch_kv<T, 256, 32>(a, append, s)
         : G == 64 ? launch_kv<T, 256, 64>(a, append, s)
                   : launch_kv<T, 256, 128>(a, append, s);
}

fgq_status run_kv(const KvArgs& a, int type, int D, int G, bool append, cudaStream_t s) {
  if (type == FGQ_F32) return launch_kv_t<float>(a, D, G, append, s);
  return type == FGQ_BF16 ? launch_kv_t<__nv_bfloat16>(a, D, G, append, s) : launch_kv_t<__half>(a, D, G, append, s);
}

// What both calls ask of their common arguments.
fgq_status check_kv(const fgq_kv_cache* cache, const void* k, const void* v, int type, int B, int T,
                    const int32_t* table, int max_pages, const int32_t* starts, const int32_t* lens) {
  if (B < 0 || T < 0 || max_pages < 0 || !valid_float(type)) return FGQ_ERR_ARG;
  const fgq_status st = check_cache(cache);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  if (!k || !v || !table || !starts) return FGQ_ERR_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(table, 4) || !aligned(starts, 4) || !aligned(lens, 4))
    return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

}  // namespace
}  // namespace fgq

using namespace fgq;

extern "C" {

fgq_status fgq_kv_append(const fgq_kv_cache* cache, const void* k, const void* v, fgq_float_type type, int B, int T,
                         int64_t k_batch_stride, int64_t k_token_stride, int64_t v_batch_stride,
                         int64_t v_token_stride, const int32_t* page_table, int max_pages, const int32_t* starts,
                         const int32_t* lens, cudaStream_t stream) {
  const fgq_status st = check_kv(cache, k, v, type, B, T, page_table, max_pages, starts, lens);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  if (!dec::stride16(k_batch_stride, type) || !dec::stride16(k_token_stride, type) ||
      !dec::stride16(v_batch_stride, type) || !dec::stride16(v_token_stride, type))
    return FGQ_ERR_ALIGN;
  KvArgs a = {};
  a.c = dec::view(cache, page_table, max_pages);
  a.k = k;
  a.v = v;
  a.bs[0] = k_batch_stride;
  a.bs[1] = v_batch_stride;
  a.ts[0] = k_token_stride;
  a.ts[1] = v_token_stride;
  a.starts = starts;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.err = device_error_word();
  return run_kv(a, type, cache->head_dim, cache->group, true, stream);
}

fgq_status fgq_kv_read(const fgq_kv_cache* cache, void* k, void* v, fgq_float_type type, int B, int T,
                       const int32_t* page_table, int max_pages, const int32_t* starts, const int32_t* lens,
                       cudaStream_t stream) {
  const fgq_status st = check_kv(cache, k, v, type, B, T, page_table, max_pages, starts, lens);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  KvArgs a = {};
  a.c = dec::view(cache, page_table, max_pages);
  a.k_out = k;
  a.v_out = v;
  a.starts = starts;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.err = device_error_word();
  return run_kv(a, type, cache->head_dim, cache->group, false, stream);
}

}  // extern "C"
